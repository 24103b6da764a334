"""What the losses' and the orthogonalised update's entry points ask for and refuse at the edges of what they document (no GPU
needed: addresses are numbers, and each call is refused)."""
import ctypes as C

import pytest

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
