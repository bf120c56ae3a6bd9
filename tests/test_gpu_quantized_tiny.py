"""Blocks whose largest magnitude lies between 2^-130 and 2^-60, where the scale's remainders reach the denormals: the definition bit
by bit (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, quantize

pytestmark = pytest.mark.gpu


def tiny_blocks(lowest, highest):
    """One block a row for each bf16 largest magnitude in the range: that over every power of two down to the denormals (448 * 2^-16
    and its neighbours lie half way between two e4m3 values), and random bf16 values under it."""
    g = np.random.default_rng(3)
    most = np.ldexp(1.0 + np.arange(128)[None, :] / 128, np.arange(lowest, highest)[:, None]).reshape(-1, 1)
    x = np.empty((len(most), BLOCK))
    x[:, :40] = np.ldexp(most, -np.arange(40)[None, :])
    x[:, 40:] = np.minimum(np.ldexp(1.0 + g.integers(0, 128, (len(most), 88)) / 128, -g.integers(0, 20, (len(most), 88))) * 2.0 ** np.floor(np.log2(most)), most)
    x *= np.where(g.random(x.shape) < 0.5, -1, 1)
    return torch.from_numpy(x).to(torch.bfloat16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lowest,highest", [(-130, -110), (-110, -90), (-90, -60)])
def test_quantize_of_tiny_blocks(lowest, highest, dtype):
    print("tiny blocks", lowest, highest, dtype, flush=True)
    x = tiny_blocks(lowest, highest)
    src = x.cuda() if dtype == "bf16" else x.float().cuda()
    q, s = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty((len(x), 1), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=len(x), cols=BLOCK, block_rows=1, dtype=bm.BM_BF16 if dtype == "bf16" else bm.BM_F32), src, q, s)
    want_q, want_s = quantize(src.float().cpu().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def test_quantize_of_tiny_matrices():
    print("tiny matrices", flush=True)
    x = tiny_blocks(-126, -96)
    x = x[::7].repeat_interleave(BLOCK, 0).view(-1, BLOCK, BLOCK)
    q, s = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty((len(x), 1, 1), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=len(x), rows=BLOCK, cols=BLOCK, block_rows=BLOCK, dtype=bm.BM_BF16), x.cuda(), q, s)
    want_q, want_s = quantize(x.float().numpy(), BLOCK)
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def test_norm_of_tiny_weights():
    """The norm's 8-bit output from its own 32-bit values, which y in fp32 shows."""
    print("tiny norm", flush=True)
    T, d = 64, 512
    g = torch.Generator().manual_seed(2)
    x = torch.randn((T, d), generator=g).cuda()
    gamma = torch.ldexp(1.0 + torch.randint(0, 128, (d,), generator=g) / 128, torch.randint(-125, -105, (d,), generator=g)).cuda()
    y, q, s = torch.empty_like(x), torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, d // BLOCK), device="cuda")
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_F32, eps=1e-6), x, None, gamma, y=y, q=q, scale=s)
    want_q, want_s = quantize(y.cpu().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)
