"""The largest sizes that the 8-bit operators take (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, quantize

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [(1 << 31) - 1, (1 << 31) - 8, (1 << 31) - 128])
def test_quantize_of_the_longest_row(cols):
    print("longest row", cols, flush=True)
    x = torch.zeros((1, cols), dtype=torch.bfloat16, device="cuda")
    head, tail = torch.randn((2, 1000), generator=torch.Generator().manual_seed(1)).bfloat16()
    x[0, :1000], x[0, cols - 1000:] = head.cuda(), tail.cuda()
    q, s = torch.full((1, cols), 0x55, dtype=torch.uint8, device="cuda"), torch.full((1, -(-cols // BLOCK)), -1.0, device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=1, cols=cols, block_rows=1, dtype=bm.BM_BF16), x, q, s)
    cut = cols - 1000 - (cols - 1000) % BLOCK                              # the first block that the tail touches
    for lo, hi in ((0, 1024), (cut, cols)):
        want_q, want_s = quantize(x[:, lo:hi].float().cpu().numpy())
        np.testing.assert_array_equal(q[:, lo:hi].cpu().numpy(), want_q)
        np.testing.assert_array_equal(s[:, lo // BLOCK:-(-hi // BLOCK)].cpu().numpy(), want_s)
    # zeros between, each with the smallest scale
    assert int(q.view(-1)[1024:cut].max()) == 0
    assert bool((s[0, 8:cut // BLOCK] == 2.0 ** -126).all())


@pytest.mark.parametrize("T,d", [((1 << 26) - 1, 8), ((1 << 25) - 1, 513), ((1 << 22) - 1, 8200)])
def test_norm_of_the_most_rows(T, d):
    """One row less than is refused: the first and the last rows, and nothing else than zeros between."""
    print("most rows", T, d, flush=True)
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    for lo in (0, T - 300):
        x[lo:lo + 300] = torch.randn((300, d), generator=g, device="cuda").bfloat16()
    w = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).bfloat16()
    y = torch.full_like(x, 7.0)
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=1e-5), x, None, w, y=y)
    for lo in (0, T - 300):
        t = x[lo:lo + 300].double()
        want = t / (t.square().mean(1, keepdim=True) + 1e-5).sqrt() * w.double()
        # bf16's half step; the 32-bit sum of squares and quotient are far below a hundredth of it
        assert bool(((y[lo:lo + 300].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs()).all())
    for part in y[300:T - 300].split(1 << 22):
        assert not bool(part.any())
