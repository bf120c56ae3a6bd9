"""Sizes at the ends of the 8-bit operators' ranges, on the host: what is past them is refused before anything is launched (CPU
only)."""
import ctypes

import pytest

import paper_2511_10054_amd as bm

ONE = ctypes.c_void_p(256)       # non-null and aligned, never dereferenced on these paths
SHAPE = -2


@pytest.mark.parametrize("n,rows,cols,block", [
    (1, 1, (1 << 31) - 1, 128), (1, 1, (1 << 31) - 127, 128),                          # 2^24 blocks a row
    (1, 17, (1 << 31) - 1, 1), (1, 16, (1 << 31) - 127, 1), (1, (1 << 28) - 15, 128, 1), (1, 1 << 27, 129, 1),      # over 2^28 - 16 blocks of rows
    (1, 65535 * 128 + 1, 1, 128), (65536, 1, 1, 128),
])
def test_quantize_refuses_grids_past_the_launch(n, rows, cols, block):
    d = bm.QuantizeDesc(n=n, rows=rows, cols=cols, block_rows=block, dtype=bm.BM_BF16)
    assert bm.load_library().bm_quantize(ctypes.byref(d), ONE, ONE, ONE, None) == SHAPE
