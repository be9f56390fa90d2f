"""Calls of more rows than one launch takes (2^32 threads in all) are refused as such, not as a failed launch after which a pool is lost (CPU)."""
import ctypes as C

import pytest

import paper_2401_06761_amd as ap

ADDRESS = 4096  # (nothing is launched)


@pytest.mark.parametrize("n,status", [(1 << 26, -6), ((1 << 26) - 3, -6), (1 << 40, -6), (-1, -1)])
def test_rotary_rows(n, status):
    L = ap.binding._L()
    with ap.Rotary(2) as rot:
        rows = ap.AparRotaryRows(ADDRESS, ADDRESS, 2, 2, 1, 2)
        assert L.apar_rotate_rows(rot.handle, ap.APAR_BF16, ADDRESS, n, rows, None, 0, None) == status


@pytest.mark.parametrize("n", [1 << 22, (1 << 31) - 1])
def test_rows_of_logits(n):
    L = ap.binding._L()
    need = C.c_size_t()
    assert L.apar_sample_workspace_bytes(n, 1, C.byref(need)) == -6
    assert L.apar_sample_tokens(ADDRESS, ap.APAR_BF16, n, 1, 1, None, ADDRESS, None, ADDRESS, None, None, 0, None) == -6
    assert L.apar_sample_workspace_bytes((1 << 22) - 1, 1, C.byref(need)) == 0
