"""What the losses' and the orthogonalised update's entry points ask for and refuse at the edges of what they document (no GPU
needed: addresses are numbers, and each call is refused)."""
import ctypes as C

import pytest
import torch

from paper_2510_11370_amd import build as hip_build
from paper_2510_11370_amd import r3

WORKSPACE = 3
A = [C.c_void_p((i + 1) << 36) for i in range(14)]


def _policy_bytes(n, nseq):
    return r3.lib().r3_policy_loss_workspace_bytes(C.byref(r3.policy_desc(n, nseq)))


@pytest.mark.parametrize("n", [0, 1, 4096, 4097, 5000, 10000, 65536, 100000, 131072, 131073, 1 << 20, (1 << 31) - 65537])
def test_a_policy_workspace_does_for_one_sequence_of_all_tokens(n):
    # without seq_start the descriptor's nseq does not count: all tokens are one sequence
    hip_build.build()
    one = _policy_bytes(n, 1)
    for nseq in (0, 1, 2, 7, 8, 9, 16, 64, 128, 129, 213, 1000, 4096, 4097, 100000):
        assert _policy_bytes(n, nseq) >= one, nseq


@pytest.mark.parametrize("n,nseq", [(5000, 16), (65536, 64), (131072, 8), (131072, 213)])
def test_the_policy_loss_refuses_a_workspace_too_small_for_one_sequence(n, nseq):
    hip_build.build()
    D = r3.policy_desc(n, nseq)
    at = A[:7] + [None] + A[8:13]                 # (no seq_start)
    assert r3.lib().r3_policy_loss(C.byref(D), *at, _policy_bytes(n, 1) - 1, None) == WORKSPACE


def _record(shape, **desc):
    D = r3.desc(6, 8, 16, 2, 8, **desc)
    rec = shape if isinstance(shape, torch.Tensor) else torch.zeros(shape, dtype=torch.uint8)
    return r3._record("call", D, rec, -1) == rec.data_ptr()


def test_the_binding_looks_at_a_record_s_rows():
    wide = torch.zeros(6, 5, dtype=torch.uint8)
    layers = torch.zeros(6, 3, 2, dtype=torch.uint8)
    # six tokens' records of two ids
    for good, stride in (((6, 2), 0), ((12,), 0), ((2, 3, 2), 0), ((9, 2), 0), (wide[:, :2], 5), (wide[:, 3:], 5), (wide, 5), ((5 * 5 + 2,), 5),
                         (layers[:, 0], 6), (layers[:, 2], 6), (layers, 6), (torch.zeros(2, 3, 4, 2, dtype=torch.uint8)[:, :, 1], 8)):
        assert _record(good, idx_token_stride=stride), (good if isinstance(good, tuple) else good.shape, stride)
    for bad, stride in ((wide[:, :2], 0), (wide, 0), (wide[:, 3:], 4), ((6, 2), 5), ((12,), 5), ((5 * 5 + 1,), 5), ((5, 2), 0), ((11,), 0), (layers[:, 0], 0), (layers, 2),
                        (layers, 0), (layers[:, :, 0], 6), (wide.T, 0), (wide[:5, :2], 5), (torch.zeros(24, dtype=torch.uint8)[::2], 0),
                        (torch.zeros(1, 2, dtype=torch.uint8).expand(6, 2), 0), (torch.zeros(6, 2, dtype=torch.uint16), 0), (torch.zeros(6, 2, dtype=torch.int64), 0)):
        with pytest.raises(r3.R3Error):
            _record(bad, idx_token_stride=stride)
    # one token: its record alone counts
    one = r3.desc(1, 8, 16, 2, 8, idx_token_stride=9)
    r3._record("call", one, torch.zeros(1, 2, dtype=torch.uint8), -1)
    with pytest.raises(r3.R3Error):
        r3._record("call", one, torch.zeros(1, 1, dtype=torch.uint8), -1)


def test_a_balance_workspace_grows_by_the_sequences_alone():
    # one layout for more than a few groups: a row of slots, of probabilities and of counts to each, whatever nseq E is modulo 2^32
    hip_build.build()
    D = r3.desc(64, 8, 256, 2, 8)
    size = lambda nseq: r3.lib().r3_balance_loss_workspace_bytes(C.byref(D), nseq)  # noqa: E731
    at = [5000, 1 << 22, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, 1 << 24, (1 << 24) + 8, 1 << 25, (1 << 31) - 65537]
    for a, b in zip(at, at[1:]):
        assert size(b) - size(a) == (b - a) * 3 * 256 * 4, (a, b)


def test_a_policy_workspace_grows_with_the_sequences_up_to_their_limit():
    hip_build.build()
    n = (1 << 31) - 65537
    at = [1 << 20, 1 << 24, 1 << 28, 1 << 30, (1 << 31) - (1 << 19), (1 << 31) - (1 << 17), (1 << 31) - 65537]
    slopes = [(_policy_bytes(n, b) - _policy_bytes(n, a)) / (b - a) for a, b in zip(at, at[1:])]
    # (four arrays, each rounded up to 256 bytes, over 2^16 sequences and more)
    assert max(slopes) - min(slopes) <= 2 * 4 * 256 / 65536, slopes


def test_the_binding_wants_three_coefficients():
    G = torch.zeros(3, 4)
    for coef in ((), (1.5,), (1.5, -0.5), (1.5, -0.5, 0.0, 0.0)):
        with pytest.raises(r3.R3Error, match="three"):
            r3.orthogonalize(G, G, coef=coef)
