"""Sizes at the ends of the 8-bit operators' ranges, on the host: what is past them is refused before anything is launched (CPU
only)."""
import ctypes
import os

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


# lanes: eight values each in whole waves of 64, at most 1024
@pytest.mark.parametrize("T,d", [(1 << 26, 1), (1 << 26, 8), (1 << 26, 512), (1 << 25, 513), (1 << 25, 1024), (1 << 22, 8192), (1 << 22, 8193), (1 << 22, 16384)])
def test_norm_refuses_grids_past_the_launch(T, d):
    desc = bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=0.0)
    assert bm.load_library().bm_add_rmsnorm(ctypes.byref(desc), ONE, ONE, ONE, None, ONE, None, None, None) == SHAPE


def test_header_states_the_norms_limit():
    """The header's text, in numbers, at both sides of what the call above refuses."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "buddymoe.h")) as f:
        text = " ".join(f.read().split())
    assert "T * lanes under 2^32, where lanes is d / 8 rounded up to whole 64s, at most 1024" in text


@pytest.mark.parametrize("over", [dict(rows=(1 << 30) + 1, a_rows=(1 << 30) + 1), dict(N=(1 << 20) + 32), dict(Kd=32800),
                                  dict(rows=1 << 24, a_rows=1 << 24, N=32 << 10, E=1), dict(rows=(1 << 24) - 8, a_rows=1 << 24, N=32 << 10, E=1)])
def test_products_refuse_grids_past_the_launch(over):
    d = bm.ProductDesc(**dict(dict(rows=8, a_rows=8, N=64, Kd=64, E=4, K=1, dtype=bm.BM_BF16), **over))
    assert bm.load_library().bm_grouped_matmul(ctypes.byref(d), *(ONE,) * 7, None) == SHAPE
    assert bm.load_library().bm_grouped_swiglu(ctypes.byref(d), *(ONE,) * 10, None) == SHAPE


@pytest.mark.parametrize("over", [
    dict(T=1 << 22, K=8, F=32768), dict(T=1 << 20, K=8, d=32768, F=32),               # products of too many tiles
    dict(T=(1 << 27) + 1, K=8), dict(T=1 << 20, K=1, d=32768),                        # rows, blocks of the tokens
])
def test_layer_of_refused_size_has_no_workspace(over):
    d = bm.LayerDesc(**dict(dict(T=16, d=64, E=8, F=64, K=2, n_shared=0, R=3, H=3, dtype=bm.BM_BF16, flags=bm.BM_RENORM_TOPK), **over))
    assert bm.bm_workspace_bytes_quantized(d) == 0
    w = bm.QuantizedWeights(*([256] * len(bm.QuantizedWeights._fields_)))
    assert bm.load_library().bm_moe_forward_quantized(ctypes.byref(d), ONE, ONE, ONE, ctypes.byref(w), ONE, ONE, ONE, ONE, 1 << 60, None, None) == SHAPE
    d.T = 64
    assert bm.bm_workspace_bytes_quantized(d) > 0
