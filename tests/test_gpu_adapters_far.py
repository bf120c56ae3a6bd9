"""Low-rank adapters whose u = A x lies beside the largest number of 16 bits (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows,rank", [(3, 16), (10, 40), (40, 16), (70, 8), (200, 33), (200, 64), (80, 128)])
def test_u_between_the_largest_bf16_and_the_largest_fp32(rows, rank, y):
    """u = +-(2 - 2^-9) 2^127, which would round to infinity in bf16, as (2 - 2^-7) 2^127 + 3 * 2^-9 * 2^127, and b = 2^-120: y = base +- 255.75,
    (256 - 2^-2) exact in fp32, rounded once in bf16."""
    import torch
    import paper_2511_10054_amd as bm
    Kd, N = 64, 96
    x = torch.zeros((rows, Kd), dtype=torch.bfloat16, device="cuda")
    x[:, 0] = x[:, 33] = 2.0 ** 100
    x[1::2] *= -1
    a = torch.zeros((2, rank, Kd), dtype=torch.bfloat16, device="cuda")
    a[1, rank - 1, 0], a[1, rank - 1, 33] = (2 - 2.0 ** -7) * 2.0 ** 27, 3 * 2.0 ** -9 * 2.0 ** 27
    b = torch.zeros((2, N, rank), dtype=torch.bfloat16, device="cuda")
    b[1, :, rank - 1] = 2.0 ** -120
    yt = torch.float32 if y == "f32" else torch.bfloat16
    base = torch.arange(N, dtype=torch.float32, device="cuda").repeat(rows, 1).to(yt)
    adapter = torch.ones(rows, dtype=torch.int32, device="cuda")
    adapter[2] = 0
    out = torch.empty_like(base)
    desc = bm.AdapterDesc(rows=rows, Kd=Kd, N=N, n=2, rank=rank, dtype=bm.BM_BF16, y_dtype=bm.BM_F32 if y == "f32" else bm.BM_BF16)
    bm.bm_add_adapters(desc, x, adapter, a, b, None, None, base, out, torch.empty(bm.bm_workspace_bytes_adapters(desc), dtype=torch.uint8, device="cuda"))
    sign = torch.ones(rows, 1, device="cuda")
    sign[1::2] = -1
    sign[2] = 0
    assert torch.equal(out, (base.float() + 255.75 * sign).to(yt))
