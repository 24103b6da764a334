"""r3_orthogonalize against oracle/operators.py (64 bits), its refusals of what it documents, and its use on the gradients of a
layer's backward."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2510_11370_amd import r3

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gradient(b, r, c, src, seed=0, kind="falling"):
    g = torch.Generator().manual_seed(seed + 1000 * b + 37 * r + c)
    low = max(1, min(r, c) // 4)
    x = torch.randn(b, r, c, generator=g) if kind == "flat" else (
        (torch.randn(b, r, low, generator=g) * torch.arange(1, low + 1).pow(-0.7)) @ torch.randn(b, low, c, generator=g)
        + 0.3 * torch.randn(b, r, c, generator=g))
    return (x * 1e-3).to(DT[src])


def _check(out, G, to, **kw):
    n = G.shape[0]
    for i in range(n) if n < 8 else (0, 1, n // 2, n - 2, n - 1):
        want, tol = ref.orthogonalize(G[i].double().numpy(), to=to, **kw)
        off = np.linalg.norm(out[i].double().cpu().numpy() - want)
        assert off <= tol, (i, off, tol, np.linalg.norm(want))


SIZES = [(1, 1, 1), (1, 1, 9), (2, 7, 1), (2, 5, 3), (3, 64, 64), (1, 128, 128), (2, 129, 130), (2, 64, 300), (1, 300, 64),
         (3, 257, 129), (1, 130, 1000), (2, 501, 260), (5, 100, 100), (1, 1, 5000), (2, 40, 2055), (1, 128, 2048), (70, 129, 200), (40, 300, 385),
         (12, 700, 520), (300, 64, 64)]


@pytest.mark.parametrize("src,to", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("b,r,c", SIZES)
def test_orthogonalize(b, r, c, src, to):
    G = _gradient(b, r, c, src)
    big = torch.full((b + 1, r, c), 77.0, dtype=DT[to], device=DEV)
    r3.orthogonalize(G.to(DEV), big[:b], scale=1.5)
    assert (big[b:] == 77).all()
    _check(big[:b], G, to, scale=1.5)


# enough of them for the large tiles, whose last ones hang over the matrices
MANY = [(110, 130, 640), (70, 300, 700), (50, 700, 400), (40, 385, 900), (64, 257, 1000), (60, 512, 512), (300, 200, 260), (9, 1100, 1300),
        (130, 130, 640), (90, 300, 700), (12, 1100, 1300)]


@pytest.mark.parametrize("src,to", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("b,r,c", MANY)
def test_many_matrices(b, r, c, src, to):
    G = _gradient(b, r, c, src, seed=1)
    big = torch.full((b + 1, r, c), 77.0, dtype=DT[to], device=DEV)
    r3.orthogonalize(G.to(DEV), big[:b], scale=1.5)
    assert (big[b:] == 77).all()
    _check(big[:b], G, to, scale=1.5)
    clean = big[:b].clone()
    G[b // 3, r - 1, c - 1] = float("nan")
    G[0] = 0.0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    r3.orthogonalize(G.to(DEV), big[:b], scale=1.5, status=status)
    assert status.item() == r3.DATA_NONFINITE and torch.isnan(big[b // 3]).all() and (big[0] == 0).all()
    rest = [i for i in range(1, b) if i != b // 3]
    assert torch.equal(big[rest], clean[rest])


# short sides of up to 128: one work-group to a matrix, two, many, and the last of them with a few columns
NARROW = [(1, 128, 64), (1, 128, 65), (1, 3, 193), (1, 1000, 65), (2, 40, 20000), (128, 100, 700), (300, 128, 520), (130, 1281, 33), (60, 900, 64), (700, 20, 30),
          (257, 2, 257), (3, 128, 8192)]


@pytest.mark.parametrize("src,to", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("b,r,c", NARROW)
def test_short_sides(b, r, c, src, to):
    G = _gradient(b, r, c, src, seed=3)
    big = torch.full((b + 1, r, c), 77.0, dtype=DT[to], device=DEV)
    for steps in (5, 1):
        r3.orthogonalize(G.to(DEV), big[:b], scale=1.5, steps=steps)
        assert (big[b:] == 77).all()
        _check(big[:b], G, to, scale=1.5, steps=steps)
    clean = big[:b].clone()
    G[b // 3, r - 1, c - 1] = float("-inf")
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    r3.orthogonalize(G.to(DEV), big[:b], scale=1.5, steps=1, status=status)
    assert status.item() == r3.DATA_NONFINITE and torch.isnan(big[b // 3]).all()
    rest = [i for i in range(b) if i != b // 3]
    assert torch.equal(big[rest], clean[rest])


def test_more_matrices_than_a_launch_has_threads_for():
    G = torch.empty(17_000_000, 1, 1, device=DEV).uniform_(0.5, 2.0).mul_(torch.where(torch.rand(17_000_000, 1, 1, device=DEV) < 0.5, -1.0, 1.0))
    out = torch.full_like(G, 7.0)
    r3.orthogonalize(G, out, steps=2)
    want, tol = ref.orthogonalize(np.ones((1, 1)), steps=2)
    # (1e-7 of 0.5 and more, by the steepest slope of two steps)
    assert ((out * G.sign() - float(want[0, 0])).abs() <= tol + 2e-7 * 12).all()


def test_what_one_step_alone_has_room_for():
    # two of these steps in one would need a matrix beyond the range of what products are made of
    G = _gradient(90, 300, 700, "f32", kind="flat")
    coef = (4.2, -14.0, 10.0)
    for to in ("f32", "bf16"):
        out = torch.empty(90, 300, 700, dtype=DT[to], device=DEV)
        r3.orthogonalize(G.to(DEV), out, steps=3, coef=coef)
        _check(out, G, to, steps=3, coef=coef)
        one = torch.empty(1, 300, 700, dtype=DT[to], device=DEV)
        r3.orthogonalize(G[:1].to(DEV), one, steps=3, coef=coef)
        _check(one, G[:1], to, steps=3, coef=coef)


@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("n", [64, 90])
def test_many_matrices_of_low_rank(n, to):
    g = torch.Generator().manual_seed(2)
    G = (torch.randn(n, 300, 3, generator=g) * torch.tensor([1.0, 0.6, 0.1])) @ torch.randn(n, 3, 700, generator=g)
    G[5] = torch.outer(torch.arange(300.0), torch.ones(700))
    out = torch.empty(n, 300, 700, dtype=DT[to], device=DEV)
    r3.orthogonalize(G.to(DEV), out)
    _check(out[4:11], G[4:11], to)


@pytest.mark.parametrize("steps", [1, 2, 3, 6, 9])
@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,c", [(2, 70, 140), (70, 300, 700), (90, 300, 700), (3, 300, 700)])
def test_steps_and_coefficients(b, r, c, steps, to):
    G = _gradient(b, r, c, "f32", seed=steps, kind="flat")
    for coef in (ref.QUINTIC, (1.5, -0.5, 0.0), (15 / 8, -10 / 8, 3 / 8)):
        out = torch.empty(b, r, c, dtype=DT[to], device=DEV)
        r3.orthogonalize(G.to(DEV), out, steps=steps, coef=coef, scale=-0.25, eps=0.0)
        _check(out, G, to, steps=steps, coef=coef, scale=-0.25, eps=0.0)
    a, b = torch.empty_like(out), torch.empty_like(out)
    r3.orthogonalize(G.to(DEV), a, steps=steps)
    r3.orthogonalize(G.to(DEV), b, steps=steps, coef=ref.QUINTIC)
    assert torch.equal(a, b)


@pytest.mark.parametrize("factor", [1e-30, 1e-12, 1e12, 1e30])
@pytest.mark.parametrize("to", ["f32", "bf16"])
def test_gradients_of_any_size(factor, to):
    G = (_gradient(2, 60, 90, "f32", kind="flat").double() * factor).float()
    out = torch.empty(2, 60, 90, dtype=DT[to], device=DEV)
    r3.orthogonalize(G.to(DEV), out, eps=0.0)
    _check(out, G, to, eps=0.0)


def test_eps_counts_against_the_norm():
    G = _gradient(1, 33, 50, "f32")
    out = torch.empty(1, 33, 50, device=DEV)
    r3.orthogonalize(G.to(DEV), out, eps=float(G.norm()))
    _check(out, G, "f32", eps=float(G.norm()))


def test_one_entry_and_low_rank():
    G = torch.zeros(3, 200, 150)
    G[0, 17, 91] = -3.0
    G[1, :, 4] = 1.0
    G[2] = torch.outer(torch.arange(200.0), torch.ones(150)) * 1e-5
    for to in ("f32", "bf16"):
        out = torch.empty(3, 200, 150, dtype=DT[to], device=DEV)
        r3.orthogonalize(G.to(DEV), out)
        _check(out, G, to)


@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_zeros_and_values_that_are_not_finite_stay_in_their_matrix(bad, to):
    G = _gradient(5, 70, 200, "f32")
    G[1] = 0.0
    clean = torch.empty(5, 70, 200, dtype=DT[to], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    r3.orthogonalize(G.to(DEV), clean, status=status)
    assert status.item() == 0 and (clean[1] == 0).all()
    r3.orthogonalize(torch.zeros(1, 3, 4, device=DEV), zero := torch.full((1, 3, 4), 7.0, device=DEV), eps=0.0)
    assert (zero == 0).all()
    G[3, 69, 199] = bad
    out = torch.empty_like(clean)
    r3.orthogonalize(G.to(DEV), out, status=status)
    assert status.item() == r3.DATA_NONFINITE
    assert torch.isnan(out[3]).all()
    for i in (0, 1, 2, 4):
        assert torch.equal(out[i], clean[i])


@pytest.mark.parametrize("to", ["f32", "bf16"])
@pytest.mark.parametrize("b,r,c", [(9, 200, 90), (9, 96, 300), (9, 640, 640), (40, 300, 700)])
def test_a_matrix_keeps_its_bits_beside_others_and_in_place(b, r, c, to):
    G = _gradient(b, r, c, to).to(DEV)
    out = torch.empty_like(G)
    r3.orthogonalize(G, out)
    again = torch.empty_like(G)
    r3.orthogonalize(G, again)
    assert torch.equal(again, out)
    H = torch.flip(G, (0,)) * 3.0
    H[b // 2] = G[b // 2]
    r3.orthogonalize(H, again)
    assert torch.equal(again[b // 2], out[b // 2])
    r3.orthogonalize(G, G)
    assert torch.equal(G, out)
