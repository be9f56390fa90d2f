"""What the compiler makes of the kernels of 4-bit pools, rotary positions and sampling: none needs scratch memory."""
import pytest

from test_device_code import _compiled


@pytest.mark.parametrize("source,n", [("kernels_attn_fp4.hip", 6), ("kernels_matrix_fp4.hip", 1), ("kernels_append_fp4.hip", 5),
                                      ("kernels_rotary.hip", 8), ("kernels_sample.hip", 5)])
def test_no_kernel_needs_scratch(tmp_path_factory, source, n):
    found = _compiled(tmp_path_factory, source)
    assert len(found) == n and all(scratch == 0 for _, scratch in found.values()), found
