"""8-bit products at the sizes where every tile shape is taken, past 32-bit offsets, captured, and on several streams, against
products of doubles (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, product_error
from test_gpu_quantized import check_swiglu

pytestmark = pytest.mark.gpu


def values_of(q, s, block_rows=1):
    """What bytes and scales stand for, in doubles on the GPU."""
    rows, cols = q.shape
    s = s.double().repeat_interleave(BLOCK, 1)[:, :cols]
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, 0)[:rows]
    return q.view(torch.float8_e4m3fn).double() * s


class Operands:
    """Random bytes (no NaN) and scales; the matrices of groups without rows are NaN.  Their products are about one."""

    def __init__(self, counts, N, Kd, a_rows, matrices=1, K=1, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + N * 31 + Kd)
        kb, nb, E = -(-Kd // BLOCK), -(-N // BLOCK), len(counts)

        def some(*shape):
            q = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
            return torch.where((q & 0x7f) == 0x7f, q ^ 0x11, q)

        def scales(size, *shape):
            return size * torch.exp(0.5 * torch.randn(shape, generator=g, device="cuda"))

        self.counts, self.N, self.Kd, self.a_rows, self.K = counts, N, Kd, a_rows, K
        self.a, self.sa = some(a_rows, Kd), scales(1 / 140, a_rows, kb)
        self.w = [(some(E, N, Kd), scales(1 / 140 / Kd ** 0.5, E, nb, kb)) for _ in range(matrices)]
        for q, s in self.w:
            for e, n in enumerate(counts):
                if n == 0:
                    q[e], s[e] = 0x7f, float("nan")
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        self.rows = int(sum(counts))
        ids = torch.randperm(a_rows * K, generator=g, device="cuda")[:self.rows]
        self.map = ids.int() if K > 1 else None
        self.src = ids // K if K > 1 else torch.arange(self.rows, device="cuda")

    def exact(self, i=0):
        """(products, their sums of magnitudes)"""
        x = values_of(self.a, self.sa)[self.src]
        c, absolute = (torch.zeros((self.rows, self.N), dtype=torch.float64, device="cuda") for _ in range(2))
        lo = 0
        for e, n in enumerate(self.counts):
            if n:
                m = values_of(self.w[i][0][e], self.w[i][1][e], BLOCK).T.contiguous()
                c[lo:lo + n], absolute[lo:lo + n] = x[lo:lo + n] @ m, x[lo:lo + n].abs() @ m.abs()
            lo += n
        return c, absolute

    def desc(self, rows, dtype=0):
        return bm.ProductDesc(rows=rows, a_rows=self.a_rows, N=self.N, Kd=self.Kd, E=len(self.counts), K=self.K, dtype=dtype)

    def mapped(self, slack):
        return None if self.map is None else torch.cat([self.map, torch.full((slack,), -1, dtype=torch.int32, device="cuda")])

    def product(self, tt, slack=0, stream=None, c=None):
        if c is None:
            c = torch.full((self.rows + slack, self.N), -7.0, dtype=tt, device="cuda")
        bm.bm_grouped_matmul(self.desc(self.rows + slack, bm.BM_F32 if tt == torch.float32 else bm.BM_BF16), self.a, self.sa, self.mapped(slack),
                             self.offsets, *self.w[0], c, stream=stream)
        return c

    def swiglu(self, slack=0, stream=None):
        h = torch.full((self.rows + slack, self.N), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.full((self.rows + slack, -(-self.N // BLOCK)), -7.0, device="cuda")
        bm.bm_grouped_swiglu(self.desc(self.rows + slack), self.a, self.sa, self.mapped(slack), self.offsets, *self.w[0], *self.w[1], h, s, stream=stream)
        return h, s


def mixed(groups, most, seed):
    """Group sizes from zero on, sixteen and its neighbours among them."""
    n = np.random.default_rng(seed).integers(0, most + 1, groups)
    n[:4] = [0, 1, 16, 17]
    return [int(v) for v in n]


SIXTY = [60, 200, 0, 1, 33, 64, 70, 52]
FORTY = [36, 0, 129, 1, 15, 16, 64, 40]
TWENTY = [24, 0, 65, 1, 15, 16, 64, 7]
# (rows a group, columns, reduction, slots of a row in a gathered input); reductions: whole blocks, an odd number of them, a cut one
PRODUCTS = [
    ([600, 700], 8224, 512, 1), ([600, 0, 700], 8224, 480, 2), ([1300], 9472, 640, 1), ([1153], 9504, 96, 4),        # 192 x 256
    (SIXTY, 3200, 512, 1), (SIXTY, 3232, 2048, 8), (SIXTY, 3200, 352, 2), ([130] * 40, 1056, 768, 1),               # 128 x 128
    ([130] * 8, 4096, 4096, 1), ([140, 0, 260, 1, 129, 128, 255, 127], 4128, 4128, 2),                             # 128 x 256 in bf16
    ([1000], 2080, 1440, 1), ([300, 280, 310, 290], 2048, 2048, 2), ([900], 2560, 512, 1), ([0, 299, 700], 2080, 96, 4),          # 128 x 128, a unit each
    (TWENTY, 3200, 512, 1), (TWENTY, 3232, 416, 4), (FORTY, 2816, 2176, 1), (FORTY, 2848, 2080, 2),                 # 64 x 128
    ([5], 160, 2048, 1), ([1], 4096, 4096, 1), ([17, 0, 33, 1], 96, 4128, 2), ([32], 512, 14336, 1),                # streamed
    ([9, 0, 1, 8], 64, 14464, 1), ([3, 12], 32, 32768, 1), ([1, 0, 2], 96, 14368, 3),                               # by eight rows
    (mixed(16, 12, 1), 800, 2048, 1), (mixed(16, 40, 2), 800, 2176, 2), (mixed(20, 20, 3), 832, 2336, 1), (mixed(16, 12, 4), 1600, 4096, 4),   # in two parts
    (mixed(64, 12, 5), 1056, 512, 1), (mixed(64, 12, 6), 1056, 768, 8), (mixed(60, 9, 7), 1184, 96, 1), (mixed(64, 9, 8), 1152, 1952, 2),      # 32 x 128
]


def a_rows_of(counts, K):
    return -(-sum(counts) // K) + (3 if K > 1 else 9)


@pytest.mark.parametrize("counts,N,Kd,K", PRODUCTS)
def test_products_in_every_tile_shape(counts, N, Kd, K):
    print("product", sum(counts), len(counts), N, Kd, K, flush=True)
    o = Operands(counts, N, Kd, a_rows_of(counts, K), K=K)
    want, absolute = o.exact()
    bound = product_error(absolute, Kd)
    c = o.product(torch.float32, slack=6).double()
    assert bool((c[o.rows:] == -7.0).all())
    worst = float(((c[:o.rows] - want).abs() / (bound + 1e-30)).max())
    assert worst <= 1.0, worst
    c = o.product(torch.bfloat16, slack=6).double()
    assert bool((c[o.rows:] == -7.0).all())
    err = (c[:o.rows] - want).abs()
    # eight products at once, each cut below 2^-13 of the largest; bf16's half step
    assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * 1.01 * absolute + bound).all())
    assert float(err.norm()) <= 2.0 ** -8 * float(want.norm())


EXPERTS = [
    ([1300], 4864, 512, 1), ([500, 0, 800], 4896, 640, 2), ([300, 400, 500], 5024, 96, 1), ([600, 710], 5024, 1184, 3),          # 192 rows
    ([300, 250, 280], 4128, 512, 1), ([300, 250, 280], 4128, 352, 6), ([70, 1, 129, 90], 7200, 4096, 2),                         # 128 rows
    ([300, 0, 700], 384, 640, 2), ([513, 140], 416, 1184, 3), ([130, 0, 300, 128], 1408, 512, 6), ([129, 200], 2080, 2048, 2),   # few tiles: 32 rows
    ([70, 1, 129], 160, 4096, 1), ([150, 90, 97], 96, 352, 1), ([1000], 1408, 736, 1),
    ([2], 1408, 4096, 1), (mixed(16, 20, 11), 768, 2048, 8), (mixed(10, 60, 12), 416, 736, 2), ([33], 128, 32768, 1),             # 32 rows, four stages
    (mixed(64, 12, 13), 1152, 512, 1), (mixed(64, 40, 14), 1056, 608, 4), (mixed(128, 6, 15), 768, 2048, 8), (mixed(60, 9, 16), 1184, 96, 1),   # two
]


@pytest.mark.parametrize("counts,N,Kd,K", EXPERTS)
def test_swiglu_in_every_tile_shape(counts, N, Kd, K):
    print("swiglu", sum(counts), len(counts), N, Kd, K, flush=True)
    o = Operands(counts, N, Kd, a_rows_of(counts, K), matrices=2, K=K)
    h, s = o.swiglu(slack=4)
    assert bool((h[o.rows:] == 0x55).all()) and bool((s[o.rows:] == -7.0).all())
    (wg, ag), (wu, au) = o.exact(0), o.exact(1)
    wg, ag, wu, au = (t.cpu().numpy() for t in (wg, ag, wu, au))
    check_swiglu(h[:o.rows].cpu().numpy(), s[:o.rows].cpu().numpy(), wg, wu, product_error(ag, Kd), product_error(au, Kd), N)


# ---- offsets past 32 bits ----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows", [40, 600, 2000])
@pytest.mark.parametrize("a_rows", [(1 << 20) - 1, 1_100_000])             # the last row short of 4 GiB (32-bit offsets) and past it
def test_gathered_rows_around_4_gib(rows, a_rows):
    print("rows around 4 GiB", rows, a_rows, flush=True)
    N, Kd = 1056 if rows < 2000 else 6272, 4096                            # (tiles of 192 rows for the most)
    o = Operands([rows], N, Kd, rows)
    a, sa = torch.empty((a_rows, Kd), dtype=torch.uint8, device="cuda"), torch.empty((a_rows, Kd // BLOCK), device="cuda")
    at = torch.linspace(a_rows - 1, 0, rows, device="cuda", dtype=torch.float64).long()
    a[at], sa[at] = o.a, o.sa
    for tt, code in ((torch.float32, bm.BM_F32), (torch.bfloat16, bm.BM_BF16)):
        c = torch.full((rows, N), float("nan"), dtype=tt, device="cuda")
        bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=a_rows, N=N, Kd=Kd, E=1, K=1, dtype=code), a, sa, at.int(), None, *o.w[0], c)
        near = o.product(tt)
        # the same tiles and the same sums
        assert torch.equal(c, near)


def test_matrices_and_results_past_4_gi_elements():
    print("matrices past 4 GiB", flush=True)
    E, N, Kd, rows = 66, 8192, 8192, 7
    o = Operands([rows], N, Kd, rows)
    w, s = torch.empty((E, N, Kd), dtype=torch.uint8, device="cuda"), torch.empty((E, N // BLOCK, Kd // BLOCK), device="cuda")
    w[E - 1], s[E - 1] = o.w[0][0][0], o.w[0][1][0]
    c = torch.full((rows, N), float("nan"), device="cuda")
    offsets = torch.tensor([0] * E + [rows], dtype=torch.int32, device="cuda")
    bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=rows, N=N, Kd=Kd, E=E, K=1, dtype=bm.BM_F32), o.a, o.sa, None, offsets, w, s, c)
    want, absolute = o.exact()
    assert bool(((c.double() - want).abs() <= product_error(absolute, Kd)).all())
    del w, s
    print("results past 4 Gi elements", flush=True)
    rows, N, Kd = 2_100_000, 2080, 32
    o = Operands([rows], N, Kd, rows)
    c = o.product(torch.bfloat16)
    for lo in (0, rows - 500):
        want = values_of(o.a[lo:lo + 500], o.sa[lo:lo + 500]) @ values_of(o.w[0][0][0], o.w[0][1][0], BLOCK).T.contiguous()
        assert float((c[lo:lo + 500].double() - want).norm()) <= 2.0 ** -8 * float(want.norm())


def test_quantize_and_norm_past_4_gi_elements():
    print("quantize past 4 Gi elements", flush=True)
    n, rows, cols = 4, 70_000, 16_384
    x = torch.zeros((n, rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((300, cols), device="cuda").bfloat16()
    x[n - 1, rows - 300:] = tail
    for block in (1, 128):
        q = torch.empty((n, rows, cols), dtype=torch.uint8, device="cuda")
        s = torch.empty((n, -(-rows // block), cols // BLOCK), device="cuda")
        bm.bm_quantize(bm.QuantizeDesc(n=n, rows=rows, cols=cols, block_rows=block, dtype=bm.BM_BF16), x, q, s)
        S = s[n - 1].repeat_interleave(block, 0)[rows - 300:rows]
        back = q[n - 1, rows - 300:].view(torch.float8_e4m3fn).double() * S.double().repeat_interleave(BLOCK, 1)
        S = S.double().repeat_interleave(BLOCK, 1)
        t = tail.double()
        assert bool(((back - t).abs() <= torch.maximum(2.0 ** -4 * t.abs(), 2.0 ** -10 * S) * 1.001).all())
        assert int(q[0].count_nonzero()) == 0
        del q, s
    print("norm past 4 Gi elements", flush=True)
    x = x.view(n * rows, cols)
    w, y = torch.ones(cols, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    bm.bm_add_rmsnorm(bm.NormDesc(T=n * rows, d=cols, dtype=bm.BM_BF16, eps=1e-5), x, None, w, y=y)
    t = tail.double()
    want = t / (t.square().mean(1, keepdim=True) + 1e-5).sqrt()
    # bf16's half step; the 32-bit sum of squares and quotient are far below a hundredth of it
    assert bool(((y[-300:].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs()).all())
    assert int(y[:1000].count_nonzero()) == 0


# ---- streams and graphs ------------------------------------------------------------------------------------------------

MIX = [([600, 700], 8224, 512, 1), (SIXTY, 3200, 512, 1), ([5], 160, 2048, 1), (mixed(16, 12, 1), 800, 2048, 1), (mixed(64, 12, 5), 1056, 512, 1)]


def test_calls_on_two_streams_at_once():
    """No state between calls: results of calls that run beside each other are those of the calls alone."""
    print("two streams", flush=True)
    sets = [Operands(c, N, Kd, a_rows_of(c, K), matrices=2, K=K, seed=i) for i, (c, N, Kd, K) in enumerate(MIX)]
    alone = [(o.product(torch.float32), o.product(torch.bfloat16), *o.swiglu()) for o in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            for o in (sets if k == 0 else sets[::-1]):
                got[k].append((o.product(torch.float32), o.product(torch.bfloat16), *o.swiglu()))
    torch.cuda.synchronize()
    for results in (got[0], got[1][::-1]):
        for one, two in zip(alone, results):
            assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_captured_operators_follow_their_inputs():
    """One graph of all operators, replayed on new inputs and group sizes, with eager work between the replays."""
    print("capture", flush=True)
    T, d, F, K, E = 96, 512, 256, 2, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    weight = torch.randn(d, generator=g, device="cuda").bfloat16()
    q, s, y = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, d // BLOCK), device="cuda"), torch.empty_like(x)
    o = Operands([24] * E, F, d, T, matrices=2, K=K)
    down = Operands([24] * E, d, F, T * K)
    h, hs = torch.empty((T * K, F), dtype=torch.uint8, device="cuda"), torch.empty((T * K, F // BLOCK), device="cuda")
    c = torch.empty((T * K, d), dtype=torch.bfloat16, device="cuda")
    whole = torch.empty((T * K, d), device="cuda")
    back_q, back_s = torch.empty((T * K, d), dtype=torch.uint8, device="cuda"), torch.empty((T * K, d // BLOCK), device="cuda")

    def run():
        bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=1e-6), x, r, weight, residual_out=r, y=y, q=q, scale=s)
        bm.bm_grouped_swiglu(bm.ProductDesc(rows=T * K, a_rows=T, N=F, Kd=d, E=E, K=K), q, s, o.map, o.offsets, *o.w[0], *o.w[1], h, hs)
        for out, code in ((c, bm.BM_BF16), (whole, bm.BM_F32)):
            bm.bm_grouped_matmul(bm.ProductDesc(rows=T * K, a_rows=T * K, N=d, Kd=F, E=E, K=1, dtype=code), h, hs, None, o.offsets, *down.w[0], out)
        bm.bm_quantize(bm.QuantizeDesc(n=1, rows=T * K, cols=d, block_rows=1, dtype=bm.BM_BF16), c, back_q, back_s)

    outs = (r, y, q, s, h, hs, c, whole, back_q, back_s)

    def fresh(i):
        gi = torch.Generator(device="cuda").manual_seed(100 + i)
        x.copy_(torch.randn((T, d), generator=gi, device="cuda"))
        r.copy_(torch.randn((T, d), generator=gi, device="cuda"))
        n = np.random.default_rng(i).multinomial(T * K, [1 / E] * E)
        o.offsets.copy_(torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32))

    fresh(0)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(1, 6):
        fresh(i)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        for t in outs[1:]:
            t.zero_()
        fresh(i)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs)), i
        assert bool(torch.isfinite(whole).all())
