"""Zeros keep their sign on the way to 8 bits: a byte is e4m3 of the quotient, -0 of a negative zero (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, quantize

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("cols", [256, 131])
def test_quantize_keeps_the_sign_of_zeros(cols, block, dtype):
    print("zeros", cols, block, dtype, flush=True)
    g = np.random.default_rng(cols)
    x = g.standard_normal((130, cols)).astype(np.float32)
    x[g.random(x.shape) < 0.3] = 0.0
    x[g.random(x.shape) < 0.3] *= -0.0                                     # either sign
    x[5], x[129] = -0.0, 0.0                                               # blocks of nothing else
    x[7, ::3] *= 1e-6                                                      # and quotients under e4m3's smallest value
    src = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    assert int((src.float().numpy().view(np.uint32) == 1 << 31).sum()) > 1000
    q = torch.empty(x.shape, dtype=torch.uint8, device="cuda")
    s = torch.empty((-(-130 // block), -(-cols // BLOCK)), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=130, cols=cols, block_rows=block, dtype=bm.BM_BF16 if dtype == "bf16" else bm.BM_F32), src.cuda(), q, s)
    want_q, want_s = quantize(src.float().numpy(), block)
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def test_norm_keeps_the_sign_of_zeros():
    print("zeros of the norm", flush=True)
    T, d = 9, 264
    g = torch.Generator().manual_seed(1)
    x = torch.randn((T, d), generator=g)
    x[:, ::4], x[3] = -0.0, -0.0
    gamma = torch.randn(d, generator=g)
    gamma[1::8] = -0.0
    y, q, s = torch.empty((T, d), device="cuda"), torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, 3), device="cuda")
    r = torch.full((T, d), -0.0, device="cuda")                            # -0 + -0 is -0; without a residual it is the zeros' sum, +0
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_F32, eps=1e-6), x.cuda(), r, gamma.cuda(), y=y, q=q, scale=s)
    assert int((y.cpu().numpy().view(np.uint32) == 1 << 31).sum()) > 100
    want_q, want_s = quantize(y.cpu().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
