"""What the layers on a given routing refuse, by the status that the header names (CPU only)."""
import ctypes

import pytest

import paper_2511_10054_amd as bm

ONE = ctypes.c_void_p(256)       # non-null and aligned, never dereferenced on these paths
SHAPE = -2


@pytest.mark.parametrize("T", [0, 16])
@pytest.mark.parametrize("buddy_q", [0, 256])
def test_token_aware_priorities_are_refused_with_and_without_their_weights(T, buddy_q):
    """They need the router's probabilities: a shape that these calls do not take, whatever the pointers."""
    lib = bm.load_library()
    desc = bm.LayerDesc(T=T, d=64, E=8, F=128, K=2, R=3, H=3, dtype=bm.BM_BF16, flags=bm.BM_PSI_TOKEN, psi_eta=1.0)
    names = [f[0] for f in bm.Weights._fields_]
    weights = bm.Weights(*[buddy_q if n == "buddy_q" else 0 if n.startswith("wp_") or n.startswith("wsp_") else 256 for n in names])
    assert lib.bm_moe_forward_routed(ctypes.byref(desc), *(ONE,) * 3, ctypes.byref(weights), *(ONE,) * 4, 1 << 40, None, None) == SHAPE
    weights = bm.QuantizedWeights(*[buddy_q if f[0] == "buddy_q" else 256 for f in bm.QuantizedWeights._fields_])
    assert lib.bm_moe_forward_routed_quantized(ctypes.byref(desc), *(ONE,) * 5, ctypes.byref(weights), *(ONE,) * 4, 1 << 40, None, None) == SHAPE
