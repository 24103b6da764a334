"""The 64-bit references of oracle/operators.py against automatic differentiation and differences, and what the operators'
entry points refuse before anything reaches a device (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2510_11370_amd import build as hip_build
from paper_2510_11370_amd import r3

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def _case(n=5, V=37, seed=0):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 3, (n, V))
    z[1, ::3] = -np.inf
    t = rng.integers(0, V, n)
    t[1] = 1
    t[2] = -1
    return z, t, rng.normal(0, 1, n), rng.normal(0, 0.3, n)


def test_log_probabilities_and_their_gradient_against_autograd():
    z, t, dl, dh = _case()
    scale = float(np.float32(1 / 0.7))
    f = ref.token_logprobs(z, t, scale, top=4)
    keep = torch.tensor(t >= 0)
    zt = torch.tensor(np.where(np.isinf(z), -1e300, z), requires_grad=True)
    lp = torch.log_softmax(scale * zt, 1)
    logp = lp.gather(1, torch.tensor(np.maximum(t, 0))[:, None])[:, 0]
    H = -(lp.exp() * torch.where(lp.exp() > 0, lp, torch.zeros_like(lp))).sum(1)
    k = keep.numpy()
    np.testing.assert_allclose(f["logp"][k], logp.detach().numpy()[k], rtol=1e-13)
    np.testing.assert_allclose(f["entropy"][k], H.detach().numpy()[k], rtol=1e-13)
    assert f["logp"][2] == f["entropy"][2] == 0 and (f["top_id"][2] == -1).all()
    best = lp.detach().topk(4, 1)
    np.testing.assert_allclose(f["top_logp"][k], best.values.numpy()[k], rtol=1e-13)
    assert np.array_equal(f["top_id"][k], best.indices.numpy()[k])
    ((torch.tensor(dl) * logp + torch.tensor(dh) * H)[keep]).sum().backward()
    dz, _ = ref.token_logprobs_backward(z, t, scale, dl, dh, 0.0)
    np.testing.assert_allclose(dz, zt.grad.numpy(), rtol=1e-12, atol=1e-14)


def test_the_gradient_of_the_logits_against_differences():
    z, t, dl, dh = _case(seed=3)
    scale, h = float(np.float32(0.8)), 1e-5

    def loss(zz):
        f = ref.token_logprobs(zz, t, scale)
        return (dl * f["logp"] + dh * f["entropy"])[t >= 0].sum()

    dz, _ = ref.token_logprobs_backward(z, t, scale, dl, dh, 0.0)
    for i, v in [(0, 0), (0, int(t[0])), (1, 0), (1, 1), (1, 2), (3, 5), (4, int(t[4]))]:
        a, b = z.copy(), z.copy()
        a[i, v] += h
        b[i, v] -= h
        assert abs((loss(a) - loss(b)) / (2 * h) - dz[i, v]) < 1e-9, (i, v)


def test_ties_masks_and_rows_of_nothing():
    z = np.array([[0.0, -0.0, 1.0, 1.0], [-np.inf] * 4, [np.nan, 0, 0, 0], [5.0, -np.inf, -np.inf, 5.0]])
    f = ref.token_logprobs(z, np.array([0, 1, 2, 1]), 1.0, top=3)
    assert f["top_id"].tolist() == [[2, 3, 0], [-1, -1, -1], [-1, -1, -1], [0, 3, -1]]
    assert f["logp"][1] == -np.inf and f["entropy"][1] == 0 and np.isnan(f["logp"][2]) and f["logp"][3] == -np.inf
    assert np.isneginf(f["top_logp"][1]).all() and np.isneginf(f["top_logp"][3, 2])


def test_gradients_of_combine_and_permute_against_autograd():
    rng = np.random.default_rng(4)
    T, K, d = 7, 3, 5
    inv = rng.permutation(T * K)
    s, Yp, x, dy, dXp = (rng.normal(size=k) for k in ((T, K), (T * K, d), (T, d), (T, d), (T * K, d)))
    st, Yt, xt = (torch.tensor(v, requires_grad=True) for v in (s, Yp, x))
    g = torch.softmax(st, 1)
    g.retain_grad()
    y = (g[:, :, None] * Yt[torch.tensor(inv)].view(T, K, d)).sum(1)
    (y * torch.tensor(dy)).sum().backward()
    got = ref.combine_backward(dy, Yp, g.detach().numpy(), inv, 0.0)
    np.testing.assert_allclose(got["dYp"], Yt.grad.numpy(), rtol=1e-13)
    np.testing.assert_allclose(got["dgates"], g.grad.numpy(), rtol=1e-12)
    np.testing.assert_allclose(got["dz"], st.grad.numpy(), rtol=1e-10, atol=1e-14)
    Xp = torch.zeros(T * K, d, dtype=torch.float64)
    Xp = Xp.index_put((torch.tensor(inv),), xt.repeat_interleave(K, 0))
    (Xp * torch.tensor(dXp)).sum().backward()
    dx, _ = ref.permute_backward(dXp, inv, None, T, 0.0)
    np.testing.assert_allclose(dx, xt.grad.numpy(), rtol=1e-13)


# ---- refusals: addresses are numbers here, nothing is launched
A = [C.c_void_p((i + 1) << 30) for i in range(12)]


def _lp(n=4, V=100, dtype=0, logits=A[0], ld=100, scale=1.0, target=A[1], logp=A[2], entropy=A[3], stats=A[4], top=2, top_logp=A[5],
        top_id=A[6], status=A[7], ws=A[8], ws_bytes=1 << 20):
    return r3.lib().r3_token_logprobs(n, V, dtype, logits, ld, scale, target, logp, entropy, stats, top, top_logp, top_id, status, ws,
                                      ws_bytes, None)


def _lb(n=4, V=100, dtype=0, logits=A[0], ld=100, scale=1.0, target=A[1], stats=A[2], entropy=A[3], dlogp=A[4], dentropy=A[5],
        dlogits=A[6], ldd=100):
    return r3.lib().r3_token_logprobs_backward(n, V, dtype, logits, ld, scale, target, stats, entropy, dlogp, dentropy, dlogits, ldd,
                                               None)


def _off(p, n):
    return C.c_void_p(p.value + n)


def test_log_probabilities_refuse():
    hip_build.build()
    for bad in (dict(n=-1), dict(V=0), dict(dtype=2), dict(logits=None), dict(ld=99), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=9e-7), dict(scale=1.1e6), dict(logits=_off(A[0], 1)), dict(dtype=1, logits=_off(A[0], 2)),
                dict(target=None), dict(top=-1), dict(top=33), dict(top_logp=None), dict(top_id=None), dict(stats=_off(A[4], 2)),
                dict(target=_off(A[1], 1)), dict(status=_off(A[7], 2)),
                dict(logp=None, entropy=None, stats=None, top=0)):
        assert _lp(**bad) == INVALID, bad
    assert _lp(n=1 << 31) == UNSUPPORTED and _lp(V=(1 << 31) - 1, ld=1 << 31) == UNSUPPORTED
    assert _lp(n=1 << 30, ld=1 << 30) == UNSUPPORTED and _lp(n=2, ld=(1 << 47) + 1) == UNSUPPORTED
    need = r3.lib().r3_token_logprobs_workspace_bytes(1, 151936, 20)
    assert need > 0 and need % 256 == 0
    cut = dict(n=1, V=151936, ld=151936, top=20)
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=_off(A[8], 128))):
        assert _lp(**cut, **bad) == WORKSPACE, bad
    assert _lp(n=0, logits=None, target=None, logp=None, ws=None) == OK
    for n, V, top in ((0, 100, 0), (-1, 100, 0), (1, 0, 0), (1, 100, 33), (1 << 31, 100, 1)):
        assert r3.lib().r3_token_logprobs_workspace_bytes(n, V, top) == 0


def test_gradient_of_the_logits_refuses():
    hip_build.build()
    for bad in (dict(n=-1), dict(V=0), dict(dtype=2), dict(logits=None), dict(ld=99), dict(ldd=99), dict(scale=0.0), dict(target=None),
                dict(stats=None), dict(entropy=None), dict(dlogp=None, dentropy=None), dict(dlogits=None), dict(dlogits=_off(A[6], 1)),
                dict(dlogp=_off(A[4], 2)),
                dict(dlogits=_off(A[0], 2)),                    # one element on
                dict(dlogits=A[0], ldd=101),                    # the same place, another stride
                dict(dlogits=_off(A[0], 2 * 399)),              # the last element alone
                dict(dlogits=_off(A[0], -2 * 399))):
        assert _lb(**bad) == INVALID, bad
    assert _lb(n=1 << 31) == UNSUPPORTED and _lb(ldd=1 << 47) == UNSUPPORTED and _lb(ld=1 << 47) == UNSUPPORTED
    assert _lb(n=0, logits=None, stats=None, dlogits=None) == OK


def test_gradients_of_combine_and_permute_refuse():
    hip_build.build()
    D = r3.desc(16, 8, 8, 2, 16, "bf16")

    def cb(D=D, dy=A[0], Yp=A[1], gates=A[2], inv=A[3], dYp=A[4], dg=A[5], dz=A[6]):
        return r3.lib().r3_combine_backward(C.byref(D), dy, Yp, gates, inv, dYp, dg, dz, None)

    def pb(D=D, dXp=A[0], inv=A[1], add=A[2], dx=A[3]):
        return r3.lib().r3_permute_backward(C.byref(D), dXp, inv, add, dx, None)

    rows = 16 * 2 * 8 * 2
    for bad in (dict(D=r3.desc(16, 8, 8, 9, 16)), dict(dy=None), dict(Yp=None), dict(gates=None), dict(inv=None),
                dict(dYp=None, dg=None, dz=None), dict(dy=_off(A[0], 8)), dict(Yp=_off(A[1], 2)), dict(dYp=_off(A[4], 4)),
                dict(dg=_off(A[5], 2)), dict(inv=_off(A[3], 1)), dict(dYp=_off(A[1], 16)), dict(dYp=_off(A[1], 16 - rows)),
                dict(dYp=A[0]), dict(dz=A[5])):
        assert cb(**bad) == INVALID, bad
    for bad in (dict(dXp=None), dict(inv=None), dict(dx=None), dict(add=_off(A[2], 8)), dict(dx=_off(A[3], 2)), dict(dx=A[0]),
                dict(dx=_off(A[0], rows - 16)), dict(add=_off(A[3], 16))):
        assert pb(**bad) == INVALID, bad
    wide = r3.desc((1 << 24) + 1, 512, 8, 1, 16, "bf16")
    assert cb(D=wide, Yp=None, dg=None, dz=None, dYp=C.c_void_p(1 << 50), dy=C.c_void_p(1 << 55)) == UNSUPPORTED
    assert pb(D=wide, dXp=C.c_void_p(1 << 50), dx=C.c_void_p(1 << 55), add=None) == UNSUPPORTED


def test_the_binding_refuses_what_the_library_cannot_see():
    z = torch.zeros(4, 100)
    t = torch.zeros(4, dtype=torch.int32)
    lp = torch.zeros(4)
    D = r3.desc(16, 8, 8, 2, 16, "f32")
    rows, tok, inv = torch.zeros(32, 8), torch.zeros(16, 8), torch.zeros(32, dtype=torch.int32)
    for call in (lambda: r3.token_logprobs(z, t, lp),                                  # not on a GPU
                 lambda: r3.token_logprobs(z.half(), t, lp),
                 lambda: r3.token_logprobs(z[0], t, lp),
                 lambda: r3.token_logprobs(z.t(), t, lp),
                 lambda: r3.token_logprobs_backward(z, t, lp, z, dlogp=lp),
                 lambda: r3.token_logprobs_backward(z, t, lp, z[:, :50], dlogp=lp),
                 lambda: r3.token_logprobs_backward(z, t, lp, z.bfloat16(), dlogp=lp),
                 lambda: r3.combine_backward(D, tok, rows, torch.zeros(16, 2), inv, dYp=rows),
                 lambda: r3.permute_backward(D, rows, inv, tok)):
        with pytest.raises(r3.R3Error):
            call()


def test_the_gradient_of_the_logits_refuses_to_write_over_what_it_reads():
    """dlogits of 4 x 100 bf16 at A[6], 800 bytes: an array that begins in its last four bytes, or ends in its first four."""
    hip_build.build()
    size = dict(target=16, stats=32, entropy=16, dlogp=16, dentropy=16)
    for name, nbytes in size.items():
        for at in (A[6], _off(A[6], 796), _off(A[6], 4 - nbytes)):
            assert _lb(**{name: at}) == INVALID, (name, at)
    # rows apart: what lies between two of them counts as theirs
    assert _lb(ldd=1000, stats=_off(A[6], 4 * 1000 * 2 - 1900)) == INVALID


def test_gradients_of_combine_and_permute_refuse_outputs_that_share_bytes():
    hip_build.build()
    D = r3.desc(16, 8, 8, 2, 16, "bf16")
    given = dict(dy=(A[0], 256), Yp=(A[1], 512), gates=(A[2], 128), inv=(A[3], 128), dYp=(A[4], 512), dg=(A[5], 128), dz=(A[6], 128))

    def cb(**at):
        p = [at.get(k, v[0]) for k, v in given.items()]
        return r3.lib().r3_combine_backward(C.byref(D), *p, None)

    for out in ("dYp", "dg", "dz"):
        for other, (at, nbytes) in given.items():
            if other == out:
                continue
            step = 16 if out == "dYp" else 4
            for where in (_off(at, nbytes - step), _off(at, step - given[out][1])) + (() if (out, other) in (("dYp", "Yp"), ("dg", "gates"), ("dz", "gates")) else (at,)):
                assert cb(**{out: where}) == INVALID, (out, other, where)
    for dx in (A[1], _off(A[1], 112), _off(A[1], -240)):
        assert r3.lib().r3_permute_backward(C.byref(D), A[0], A[1], A[2], dx, None) == INVALID, dx


def test_log_probabilities_refuse_outputs_that_share_bytes():
    hip_build.build()
    n, V, top = 2, 140001, 5
    need = r3.lib().r3_token_logprobs_workspace_bytes(n, V, top)
    call = dict(n=n, V=V, ld=V + 7, top=top, ws_bytes=need)
    size = dict(logp=8, entropy=8, stats=16, top_logp=40, top_id=40, status=4, ws=need, target=8, logits=(V + 7 + V) * 2)
    place = dict(logits=A[0], target=A[1], logp=A[2], entropy=A[3], stats=A[4], top_logp=A[5], top_id=A[6], status=A[7], ws=A[8])
    assert need > 0 and need % 256 == 0
    for out in ("logp", "entropy", "stats", "top_logp", "top_id", "status"):
        for other, at in place.items():
            if other != out:
                for where in (at, _off(at, size[other] - 4 & ~3), _off(at, 4 - size[out])):
                    assert _lp(**call, **{out: where}) == INVALID, (out, other, where)
    for other in ("logits", "target"):
        assert _lp(**call, ws=place[other]) == INVALID, other


def test_gradients_of_combine_and_permute_do_not_look_at_the_record():
    """Flags, id type and stride of the record that the call has no use for: what is wrong with this one is its size alone."""
    hip_build.build()
    far = [C.c_void_p((i + 1) << 50) for i in range(4)]
    for more in (dict(), dict(flags=r3.FLAG_GATED_H), dict(flags=64), dict(idx=7), dict(idx_token_stride=1), dict(idx_token_stride=-5)):
        D = r3.desc((1 << 24) + 1, 512, 8, 2, 16, "bf16")
        for k, v in more.items():
            setattr(D, k, v)
        assert r3.lib().r3_combine_backward(C.byref(D), far[0], None, far[1], far[2], far[3], None, None, None) == UNSUPPORTED, more
        assert r3.lib().r3_permute_backward(C.byref(D), far[0], far[1], None, far[2], None) == UNSUPPORTED, more
