"""Which layers of odd sizes have their operands copied, as the workspace says (no GPU needed)."""
import ctypes

import pytest

from paper_2406_05546_amd import dense


def workspace(dtype, rows, fin, fout, backward):
    l = dense.ps_linear(dtype, 0, rows, fin, fout, 1, 1, None, None)
    n = ctypes.c_uint64(0)
    assert dense._library().ps_linear_workspace_bytes(ctypes.byref(l), backward, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("dtype,size", [(dense.PS_F32, 4), (dense.PS_BF16, 2), (dense.PS_F16, 2)])
def test_copies(dtype, size):
    # large layers with odd rows, forward x and w, backward one of them and dz at least
    assert workspace(dtype, 8192, 1111, 2777, 0) >= size * 1111 * (8192 + 2777)
    assert workspace(dtype, 8192, 1111, 2777, 1) >= size * 8192 * (1111 + 2777)
    # none where rows are multiples of 16 bytes, and none for few rows of large matrices
    assert workspace(dtype, 8192, 1112, 2776, 0) < size * 1112 * 2776
    for backward in (0, 1):
        assert workspace(dtype, 1, 4097, 4099, backward) < size * 4097 * 4099
