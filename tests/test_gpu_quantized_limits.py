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
