"""The 64-bit references of the policy loss, the load-balance loss and the orthogonalised update against automatic
differentiation, differences and the singular value decomposition, and what the entry points refuse (no GPU needed)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2510_11370_amd import build as hip_build
from paper_2510_11370_amd import r3

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def _policy(n=60, seed=0):
    rng = np.random.default_rng(seed)
    logp = -np.abs(rng.normal(0, 2, n))
    old = logp + rng.normal(0, 0.4, n)
    return dict(logp=logp, old=old, infer=old + rng.normal(0, 0.4, n), ref=logp + rng.normal(0, 0.5, n), entropy=np.abs(rng.normal(0, 1, n)),
                adv=rng.normal(0, 1, n), target=np.where(rng.random(n) < 0.3, -1, 5), starts=np.array([3, 20, 20, 50, n - 4]))


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("norm", ["tokens", "sequences", "sum"])
def test_the_policy_loss_against_autograd(ratio, norm):
    a = _policy()
    kw = dict(clip_low=0.25, clip_high=0.5, dual_clip=2.0, weight_cap=1.25, kl_coef=0.125, entropy_coef=0.0625, scale=0.5)   # f32 numbers
    got = ref.policy_loss(**a, ratio=ratio, norm=norm, **kw)
    x, H = torch.tensor(a["logp"], requires_grad=True), torch.tensor(a["entropy"], requires_grad=True)
    t = {k: torch.tensor(a[k]) for k in ("old", "infer", "ref", "adv")}
    live = torch.tensor(a["target"] >= 0)
    groups = [torch.arange(b, e)[live[b:e]] for b, e in zip(a["starts"], a["starts"][1:])]
    N, S = sum(len(g) for g in groups), sum(len(g) > 0 for g in groups)
    loss = 0.0
    for g in groups:
        if len(g) == 0:
            continue
        d = x[g] - t["old"][g]
        r = (d.mean().expand(len(g)) if ratio == "sequence" else d).exp()
        A = t["adv"][g]
        gain = torch.minimum(r * A, r.clamp(0.75, 1.5) * A)
        gain = torch.where(A < 0, torch.maximum(gain, 2.0 * A), gain)
        q = t["ref"][g] - x[g]
        l = -(t["old"] - t["infer"])[g].exp().clamp(max=1.25) * gain + 0.125 * (q.exp() - 1 - q) - 0.0625 * H[g]
        loss = loss + 0.5 * l.sum() / {"tokens": N, "sequences": S * len(g), "sum": 1}[norm]
    loss.backward()
    np.testing.assert_allclose(got["stats"][0], loss.item(), rtol=1e-13)
    np.testing.assert_allclose(got["dlogp"], x.grad.numpy(), rtol=1e-12, atol=1e-15)
    np.testing.assert_allclose(got["dentropy"], H.grad.numpy(), rtol=1e-13)
    assert got["stats"][6] == N and got["stats"][7] == S and (ratio == "sequence" or 0 < got["stats"][4] < 1)
    np.testing.assert_allclose(got["stats"][0], got["stats"][1] + 0.5 * (0.125 * got["stats"][2] - 0.0625 * got["stats"][3]), rtol=1e-12)


def test_the_balance_loss_against_autograd_and_differences():
    rng = np.random.default_rng(1)
    T, E, K = 30, 7, 2
    z = rng.normal(0, 1.5, (T, E))
    z[:, 2] = -np.inf
    idx = np.argsort(-z - rng.gumbel(0, 0.5, (T, E)), 1)[:, :K]
    starts = np.array([2, 12, 12, 25])
    got = ref.balance_loss(z, idx, starts, 0.25, 0.125)
    t = torch.tensor(np.where(np.isinf(z), -1e300, z), requires_grad=True)
    bal, zl = 0.0, 0.0
    for b, e in ((2, 12), (12, 25)):
        f = torch.tensor(np.bincount(idx[b:e].reshape(-1), minlength=E) * E / (K * (e - b)))
        bal = bal + (f * torch.softmax(t[b:e], 1).mean(0)).sum() / 2
        zl = zl + (torch.logsumexp(t[b:e], 1) ** 2).sum() / 23
    loss = 0.25 * bal + 0.125 * zl
    loss.backward()
    np.testing.assert_allclose(got["stats"], [loss.item(), bal.item(), zl.item()], rtol=1e-13)
    np.testing.assert_allclose(got["dlogits"], t.grad.numpy(), rtol=1e-11, atol=1e-16)
    assert got["counts"].sum() == 23 * K and (got["counts"][1] == 0).all() and (got["probs"][1] == 0).all()
    np.testing.assert_allclose(got["probs"].sum(1), [1, 0, 1], rtol=1e-13)
    h = 1e-6
    for i, e in ((2, 0), (13, 3), (24, 6)):
        v = []
        for s in (h, -h):
            y = z.copy()
            y[i, e] += s
            v.append(ref.balance_loss(y, idx, starts, 0.25, 0.125)["stats"][0])
        assert abs((v[0] - v[1]) / (2 * h) - got["dlogits"][i, e]) < 1e-9
    # a batch routed evenly, and one routed to the experts that its router likes
    even = ref.balance_loss(np.zeros((8, 4)), np.arange(8)[:, None] % 4, None, 1.0)
    assert abs(even["stats"][1] - 1) < 1e-15 and np.abs(even["dlogits"]).max() < 1e-16


@pytest.mark.parametrize("r,c", [(5, 9), (9, 5), (6, 6), (1, 4)])
def test_the_orthogonalised_update_against_the_singular_value_decomposition(r, c):
    rng = np.random.default_rng(r * 10 + c)
    G = rng.normal(size=(r, c))
    a, b, cc = (float(np.float32(v)) for v in ref.QUINTIC)
    U, s, V = np.linalg.svd(G, full_matrices=False)
    s = s / (np.linalg.norm(G) + float(np.float32(1e-7)))
    for _ in range(5):
        s = a * s + b * s ** 3 + cc * s ** 5
    got, tol = ref.orthogonalize(G, scale=2.0)
    assert np.linalg.norm(got - 2.0 * (U * s) @ V) < 1e-12 < tol < 1e-4 * np.linalg.norm(got)
    assert ref.orthogonalize(G, to="bf16")[1] < 0.1 and (ref.orthogonalize(np.zeros((r, c)))[0] == 0).all()


def test_where_the_quintic_takes_singular_values():
    """What the header says of the default coefficients."""
    x = y = np.logspace(math.log10(0.002), 0, 200001)
    for _ in range(5):
        y = 3.4445 * y - 4.775 * y ** 3 + 2.0315 * y ** 5
    assert 0.68 < y.min() and y.max() < 1.21


# ---- refusals: addresses are numbers here, nothing is launched
A = [C.c_void_p((i + 1) << 36) for i in range(14)]
NAN, INF = float("nan"), float("inf")


def _off(p, n):
    return C.c_void_p(p.value + n)


P_ARGS = ("logp", "old", "infer", "ref", "entropy", "adv", "target", "start", "dlogp", "dentropy", "stats", "status", "ws")


def _pl(n=1000, nseq=4, ws_bytes=1 << 24, desc=None, **over):
    d = dict(ratio="token", norm="tokens", kl_coef=0.1, entropy_coef=0.1)
    at = dict(zip(P_ARGS, A))
    for k, v in over.items():
        (at if k in at else d)[k] = v
    raw = {k: d.pop(k) for k in ("ratio_code", "norm_code", "flags") if k in d}
    D = r3.policy_desc(n, nseq, **d)
    for k, f in (("ratio_code", "ratio"), ("norm_code", "norm"), ("flags", "flags")):
        if k in raw:
            setattr(D, f, raw[k])
    return r3.lib().r3_policy_loss(C.byref(D), *[at[k] for k in P_ARGS], ws_bytes, None)


def test_the_policy_loss_refuses():
    hip_build.build()
    for bad in (dict(n=-1), dict(nseq=-1), dict(nseq=0), dict(ratio_code=2), dict(ratio_code=-1), dict(norm_code=3), dict(norm_code=-1), dict(flags=2),
                dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=NAN), dict(clip_high=-0.1), dict(clip_high=INF), dict(clip_high=NAN),
                dict(dual_clip=1.0), dict(dual_clip=-2.0), dict(dual_clip=INF), dict(dual_clip=NAN), dict(weight_cap=0.0), dict(weight_cap=NAN),
                dict(kl_coef=NAN), dict(kl_coef=INF), dict(entropy_coef=INF), dict(scale=NAN), dict(logp=None), dict(adv=None), dict(stats=None),
                dict(ref=None), dict(entropy=None)):
        assert _pl(**bad) == INVALID, bad
    for k in P_ARGS[:-1]:
        assert _pl(**{k: _off(A[P_ARGS.index(k)], 2)}) == INVALID, k
    assert _pl(n=(1 << 31) - 65536) == UNSUPPORTED and _pl(nseq=(1 << 31) - 2) == UNSUPPORTED
    need = r3.lib().r3_policy_loss_workspace_bytes(C.byref(r3.policy_desc(1000, 4)))
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=_off(A[12], 128))):
        assert _pl(**bad) == WORKSPACE, bad
    assert r3.lib().r3_policy_loss_workspace_bytes(C.byref(r3.policy_desc(-1))) == 0
    assert r3.lib().r3_policy_loss(None, *A[:13], 1 << 24, None) == INVALID


def test_the_policy_loss_refuses_outputs_that_share_bytes():
    hip_build.build()
    need = r3.lib().r3_policy_loss_workspace_bytes(C.byref(r3.policy_desc(1000, 4)))
    size = {k: 4000 for k in P_ARGS}
    size.update(start=20, stats=32, status=4, ws=need)
    for adv_seq in (False, True):
        size["adv"] = 16 if adv_seq else 4000
        for out in ("dlogp", "dentropy", "stats", "status", "ws"):
            for other in P_ARGS:
                if other == out:
                    continue
                at = A[P_ARGS.index(other)]
                step = 256 if out == "ws" else 4
                for where in (at, _off(at, (size[other] - 1) // step * step), _off(at, step - (size[out] + step - 1) // step * step)):
                    assert _pl(adv_seq=adv_seq, **{out: where}) == INVALID, (out, other, where)


def _bl(T=100, E=16, K=2, logits=A[0], ld=16, idx=A[1], start=A[2], nseq=3, alpha=0.01, zeta=0.01, counts=A[3], probs=A[4], stats=A[5], dlogits=A[6], ldd=16,
        status=A[7], ws=A[8], ws_bytes=1 << 24, **desc):
    D = r3.desc(T, 8, E, K, 8, **desc)
    return r3.lib().r3_balance_loss(C.byref(D), logits, ld, idx, start, nseq, alpha, zeta, counts, probs, stats, dlogits, ldd, status, ws, ws_bytes, None)


def test_the_balance_loss_refuses():
    hip_build.build()
    for bad in (dict(T=0), dict(T=-1), dict(K=0), dict(K=17), dict(logits=None), dict(idx=None), dict(stats=None), dict(ld=15), dict(ldd=15), dict(nseq=0),
                dict(start=None), dict(nseq=-1), dict(alpha=NAN), dict(alpha=INF), dict(zeta=INF), dict(idx_token_stride=1), dict(logits=_off(A[0], 2)),
                dict(start=_off(A[2], 2)), dict(counts=_off(A[3], 1)), dict(probs=_off(A[4], 2)), dict(stats=_off(A[5], 2)), dict(dlogits=_off(A[6], 2)),
                dict(status=_off(A[7], 1)), dict(idx_dtype=torch.uint16, idx=_off(A[1], 1))):
        assert _bl(**bad) == INVALID, bad
    assert _bl(E=5000, ld=5000, ldd=5000) == UNSUPPORTED and _bl(E=300, ld=300, ldd=300, idx_dtype=torch.uint8) == UNSUPPORTED
    assert _bl(ld=1 << 42) == UNSUPPORTED and _bl(ldd=1 << 42) == UNSUPPORTED and _bl(idx_token_stride=1 << 42) == UNSUPPORTED
    D = r3.desc(100, 8, 16, 2, 8)
    need = r3.lib().r3_balance_loss_workspace_bytes(C.byref(D), 3)
    assert need > 0 and need % 256 == 0 and r3.lib().r3_balance_loss_workspace_bytes(C.byref(D), -1) == 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=_off(A[8], 64))):
        assert _bl(**bad) == WORKSPACE, bad


def test_the_balance_loss_refuses_outputs_that_share_bytes():
    hip_build.build()
    need = r3.lib().r3_balance_loss_workspace_bytes(C.byref(r3.desc(100, 8, 16, 2, 8)), 3)
    size = dict(logits=6400, idx=200, start=16, counts=192, probs=192, stats=12, dlogits=6400, status=4, ws=need)
    place = dict(logits=A[0], idx=A[1], start=A[2], counts=A[3], probs=A[4], stats=A[5], dlogits=A[6], status=A[7], ws=A[8])
    for out in ("counts", "probs", "stats", "dlogits", "status", "ws"):
        for other, at in place.items():
            if other == out:
                continue
            step = 256 if out == "ws" else 4
            for where in (at, _off(at, (size[other] - 1) // step * step), _off(at, step - (size[out] + step - 1) // step * step)):
                if (out, other) == ("dlogits", "logits") and where is at:
                    continue          # that place is allowed
                assert _bl(**{out: where}) == INVALID, (out, other, where)
    assert _bl(dlogits=A[0], ldd=17) == INVALID


def _or(batch=3, rows=20, cols=30, src=1, G=A[0], to=1, out=A[1], steps=5, coef=None, eps=1e-7, scale=1.0, status=A[2], ws=A[3], ws_bytes=1 << 30):
    return r3.lib().r3_orthogonalize(batch, rows, cols, src, G, to, out, steps, None if coef is None else (C.c_float * 3)(*coef), eps, scale, status, ws,
                                     ws_bytes, None)


def test_orthogonalize_refuses():
    hip_build.build()
    for bad in (dict(batch=-1), dict(rows=0), dict(cols=-3), dict(src=2), dict(to=-1), dict(G=None), dict(out=None), dict(steps=0), dict(steps=65), dict(eps=-1.0),
                dict(eps=NAN), dict(eps=INF), dict(scale=NAN), dict(scale=INF), dict(coef=(NAN, 0, 0)), dict(coef=(1, INF, 0)), dict(G=_off(A[0], 2)),
                dict(out=_off(A[1], 2)), dict(src=0, G=_off(A[0], 1)), dict(status=_off(A[2], 2))):
        assert _or(**bad) == INVALID, bad
    for bad in (dict(rows=32769), dict(cols=32769), dict(batch=1 << 31), dict(batch=1 << 30, rows=32768, cols=32768),
                dict(coef=(16.0, 0.0, 0.0)), dict(coef=(3.0, 0.0, 0.0)), dict(coef=(-30.0, 4.0, 2.0), steps=1), dict(coef=(1.0, 200.0, -201.0), steps=1)):
        assert _or(**bad) == UNSUPPORTED, bad
    for to in (0, 1):
        need = r3.lib().r3_orthogonalize_workspace_bytes(3, 20, 30, to)
        assert need > 0 and need % 256 == 0
        for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=_off(A[3], 16))):
            assert _or(to=to, **bad) == WORKSPACE, bad
    assert _or(batch=0, G=None, out=None, ws=None) == OK
    for args in ((0, 5, 5, 1), (1, 0, 5, 1), (1, 5, -1, 1), (1, 5, 5, 2), (1, 40000, 5, 1)):
        assert r3.lib().r3_orthogonalize_workspace_bytes(*args) == 0
    # the workspace does not grow with the batch for ever
    assert r3.lib().r3_orthogonalize_workspace_bytes(100000, 768, 2048, 1) < 6 << 30


def test_orthogonalize_refuses_outputs_that_share_bytes():
    hip_build.build()
    need = r3.lib().r3_orthogonalize_workspace_bytes(3, 20, 30, 1)
    n = 3 * 20 * 30 * 4
    size, place = dict(G=n, out=n, status=4, ws=need), dict(G=A[0], out=A[1], status=A[2], ws=A[3])
    for out in ("out", "status", "ws"):
        for other, at in place.items():
            if other == out:
                continue
            step = 256 if out == "ws" else 4
            for where in (at, _off(at, (size[other] - 1) // step * step), _off(at, step - (size[out] + step - 1) // step * step)):
                if (out, other) == ("out", "G") and where is at:
                    continue          # that place is allowed
                assert _or(**{out: where}) == INVALID, (out, other, where)
    assert _or(out=A[0], to=0) == INVALID


def test_the_binding_refuses_what_the_library_cannot_see():
    f, i = torch.zeros(8), torch.zeros(8, dtype=torch.int32)
    D, z = r3.policy_desc(8), torch.zeros(8, 4)
    L = r3.desc(8, 4, 4, 2, 4)
    for call in (lambda: r3.policy_loss(D, f, f, f),                                       # not on a GPU
                 lambda: r3.balance_loss(L, z, torch.zeros(8, 2, dtype=torch.uint8), f[:3]),
                 lambda: r3.orthogonalize(z, z),
                 lambda: r3.orthogonalize(f, f),
                 lambda: r3.orthogonalize(z.double(), z.double()),
                 lambda: r3.orthogonalize_workspace(z.half(), z)):
        with pytest.raises(r3.R3Error):
            call()
    with pytest.raises(KeyError):
        r3.policy_desc(8, ratio="word")
    assert i.dtype is torch.int32
