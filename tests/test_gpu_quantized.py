"""The 8-bit operators against numpy in 64 bits (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, TINY, bf16, decode, encode, product_error, quantize, silu, spread, tensor, values

pytestmark = pytest.mark.gpu

DT = {"bf16": (bm.BM_BF16, torch.bfloat16, 2.0 ** -8), "f32": (bm.BM_F32, torch.float32, 2.0 ** -24)}   # code, torch type, half a step


def shifted(t, by):
    """The same values `by` elements past a 16-byte boundary, poison around them."""
    if t is None or not by:
        return t
    room = torch.full((t.numel() + 32,), 0x7f if t.dtype == torch.uint8 else float("nan"), dtype=t.dtype, device=t.device)
    room[by:by + t.numel()] = t.flatten()
    return room[by:by + t.numel()].view(t.shape)


# ---- quantize --------------------------------------------------------------------------------------------------------

Q_SHAPES = [(1, 1, 1), (1, 1, 128), (1, 3, 129), (1, 5, 96), (2, 7, 1000), (1, 130, 264), (3, 129, 257), (1, 257, 8), (1, 1, 4096), (2, 128, 384)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("n,rows,cols", Q_SHAPES)
@pytest.mark.parametrize("by", [0, 1])
def test_quantize_is_the_definition_bit_by_bit(n, rows, cols, block, dtype, by):
    print("quantize", n, rows, cols, block, dtype, by, flush=True)
    g = np.random.default_rng(rows * 1000 + cols)
    x = g.standard_normal((n, rows, cols)) * np.exp(3 * g.standard_normal((n, rows, 1)))
    x[:, : rows // 2, : cols // 3] = 0.0                                    # whole blocks of zeros, and parts
    code, tt, _ = DT[dtype]
    src = torch.from_numpy(x).to(tt)
    q = torch.full((n, rows, cols), 0x55, dtype=torch.uint8, device="cuda")
    scale = torch.full((n, -(-rows // block), -(-cols // BLOCK)), -1.0, device="cuda")
    qv, sv = shifted(q, by), shifted(scale, by)
    bm.bm_quantize(bm.QuantizeDesc(n=n, rows=rows, cols=cols, block_rows=block, dtype=code), shifted(src.cuda(), by), qv, sv)
    want_q, want_s = quantize(src.float().numpy(), block)
    np.testing.assert_array_equal(sv.cpu().numpy(), want_s)
    np.testing.assert_array_equal(qv.cpu().numpy(), want_q)


@pytest.mark.parametrize("block", [1, 128])
def test_quantize_of_extreme_values(block):
    """Blocks of the smallest and the largest magnitudes keep their order; one infinity or NaN makes its block NaN, and no other."""
    print("extreme values", block, flush=True)
    x = np.zeros((4, 640), np.float32)
    x[0, :128] = np.float32(1e-45) * np.arange(128)                        # denormals under the smallest scale
    x[0, 128:256] = np.float32(3.4e38) * np.linspace(-1, 1, 128, dtype=np.float32)
    x[0, 256:384] = 1.0
    x[1, 300] = np.inf
    x[2, 400] = np.nan
    x[3, 639] = -np.inf
    q, scale = torch.zeros((4, 640), dtype=torch.uint8, device="cuda"), torch.zeros((4 if block == 1 else 1, 5), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=4, cols=640, block_rows=block, dtype=bm.BM_F32), tensor(x), q, scale)
    want_q, want_s = quantize(x, block)
    np.testing.assert_array_equal(scale.cpu().numpy(), want_s)
    bad = np.isnan(spread(want_s, 4, 640, block if block > 1 else 1))
    got = q.cpu().numpy()
    assert np.isnan(decode(got)[bad]).all() and not np.isnan(decode(got)[~bad]).any()
    np.testing.assert_array_equal(got[~bad], want_q[~bad])


# ---- norm ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 1), (1, 4096), (3, 127), (2, 128), (5, 520), (17, 1440), (1, 16384), (2, 16383), (33, 64), (4, 8200)])
@pytest.mark.parametrize("by", [0, 1])
def test_add_rmsnorm(T, d, dtype, by):
    print("norm", T, d, dtype, by, flush=True)
    code, tt, half = DT[dtype]
    g = np.random.default_rng(d)
    x, r, w = (torch.from_numpy(a).to(tt) for a in (g.standard_normal((T, d)), 3 * g.standard_normal((T, d)), 1 + 0.2 * g.standard_normal(d)))
    eps = 1e-5
    R = x.double().numpy() + r.double().numpy()
    n = R / np.sqrt((R * R).mean(1, keepdims=True) + eps) * w.double().numpy()
    out, y = (torch.full((T, d), float("nan"), dtype=tt, device="cuda") for _ in range(2))
    q, s = torch.full((T, d), 0x7f, dtype=torch.uint8, device="cuda"), torch.full((T, -(-d // BLOCK)), float("nan"), device="cuda")
    out, y, q, s = (shifted(t, by) for t in (out, y, q, s))
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=code, eps=eps), shifted(x.cuda(), by), shifted(r.cuda(), by), shifted(w.cuda(), by), out, y, q, s)
    # r: one addition in 32 bits, one rounding.  n: r's rounding twice (itself, and through the square root of the mean of
    # squares, whose sum of non-negative terms is off by at most d / 64 + 16 + 8 steps of a lane's chain and the tree, halved by
    # the root), the quotient, root and two products: five more.
    e32 = 2.0 ** -24
    en = (2 + (d / 64 + 24) / 2 + 5) * e32
    assert (np.abs(out.double().cpu().numpy() - R) <= (half + 2 * e32) * np.abs(R) + 1e-40).all()
    assert (np.abs(y.double().cpu().numpy() - n) <= (half + 1.01 * en + e32 * np.abs(x.double().numpy()) / np.maximum(np.abs(R), 1e-30)) * np.abs(n) + 1e-30).all()
    # the scale of a block: its largest value's error and one quotient; q: half a step of e4m3 (a sixteenth, 2^-10 below the
    # normal range) of the value over the scale, and the value's own error
    _, want_s = quantize(n.astype(np.float32))
    np.testing.assert_allclose(s.cpu().numpy(), want_s, rtol=2 * (en + 3 * e32))
    S = spread(s.double().cpu().numpy(), T, d, 1)
    err = np.abs(decode(q.cpu().numpy()) * S - n)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(n), 2.0 ** -10 * S) * 1.001 + 4 * en * np.abs(n)).all()


def test_add_rmsnorm_parts_and_places():
    """Any output alone, no residual, outputs over inputs: the same bits as all outputs apart."""
    T, d = 9, 1056
    g = torch.Generator().manual_seed(3)
    x, r, w = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((T, d), (T, d), (d,)))
    desc = bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=0.0)
    full = dict(residual_out=torch.empty_like(x), y=torch.empty_like(x), q=torch.empty((T, d), dtype=torch.uint8, device="cuda"),
                scale=torch.empty((T, 9), device="cuda"))
    bm.bm_add_rmsnorm(desc, x, r, w, **full)
    for keys in (("residual_out",), ("y",), ("q", "scale")):
        part = {k: torch.zeros_like(full[k]) for k in keys}
        bm.bm_add_rmsnorm(desc, x, r, w, **part)
        assert all(torch.equal(part[k], full[k]) for k in keys), keys
    x2, r2 = x.clone(), r.clone()
    bm.bm_add_rmsnorm(desc, x2, r2, w, residual_out=r2, y=x2)
    assert torch.equal(r2, full["residual_out"]) and torch.equal(x2, full["y"])
    zero, none = torch.empty_like(x), torch.empty_like(x)
    bm.bm_add_rmsnorm(desc, x, torch.zeros_like(x), w, y=zero)
    bm.bm_add_rmsnorm(desc, x, None, w, y=none)
    assert torch.equal(zero, none)


# ---- products --------------------------------------------------------------------------------------------------------


def grouped(counts, g, live_experts=None):
    """Offsets of groups with so many rows."""
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def inputs(counts, N, Kd, seed, a_rows=None, matrices=1):
    """8-bit rows and matrices; the matrices of empty groups are NaN throughout (nothing may read them)."""
    g = np.random.default_rng(seed)
    E, rows = len(counts), int(sum(counts))
    a_rows = rows if a_rows is None else a_rows
    a = quantize(g.standard_normal((a_rows, Kd)) * np.exp(g.standard_normal((a_rows, 1))))
    ws = []
    for _ in range(matrices):
        q, s = quantize(g.standard_normal((E, N, Kd)) / np.sqrt(Kd) * np.exp(g.standard_normal((E, 1, 1))), BLOCK)
        for e in range(E):
            if counts[e] == 0:
                q[e], s[e] = 0x7f, np.nan
        ws.append((q, s))
    return a, ws


def exact_products(a, w, offsets, src):
    """(c, sum |a w|) in 64 bits, rows in group order."""
    x = values(*a)[src]
    c, absolute = np.zeros((len(src), w[0].shape[1])), np.zeros((len(src), w[0].shape[1]))
    for e in range(len(offsets) - 1):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:
            m = values(w[0][e], w[1][e], BLOCK)
            c[lo:hi], absolute[lo:hi] = x[lo:hi] @ m.T, np.abs(x[lo:hi]) @ np.abs(m).T
    return c, absolute


# group sizes (0 and 1, both sides of 16, 64, 128 and 256), output width, reduction (below, on and past blocks of 128)
P_CASES = [
    ([1], 32, 32), ([3, 0, 2], 64, 96), ([17, 1, 0, 64], 96, 128), ([65, 0, 15], 256, 160), ([16, 33], 288, 1152), ([0, 0, 5], 128, 4128),
    ([1, 1, 1, 1, 1, 1, 1, 1], 416, 768), ([300, 0, 120], 320, 416), ([129, 256, 257], 512, 256), ([513, 140], 160, 1184), ([700], 2080, 1440),
    ([200, 900, 1, 0, 63], 768, 2048), ([130] * 9, 96, 224), ([2, 126, 127, 128, 255, 511], 1408, 512),
]


def run_matmul(counts, N, Kd, out, seed, slack=0, mapped=0, by_stream=None):
    """(result with `slack` rows behind the last group, exact, bound).  mapped: slots per token of a gathered input."""
    g = np.random.default_rng(seed + 1)
    offsets = grouped(counts, g)
    rows = int(offsets[-1])
    K = max(mapped, 1)
    a_rows = max(1, -(-rows // K)) if mapped else rows + slack
    a, (w,) = inputs(counts, N, Kd, seed, a_rows)
    perm = np.concatenate([g.permutation(a_rows * K)[:rows], np.full(slack, -1)]).astype(np.int32) if mapped else None
    src = perm[:rows] // K if mapped else np.arange(rows)
    c = torch.full((rows + slack, N), -7.0, dtype=DT[out][1], device="cuda")
    bm.bm_grouped_matmul(bm.ProductDesc(rows=rows + slack, a_rows=a_rows, N=N, Kd=Kd, E=len(counts), K=K, dtype=DT[out][0]),
                         tensor(a[0]), tensor(a[1]), None if perm is None else tensor(perm), tensor(offsets), tensor(w[0]), tensor(w[1]), c)
    want, absolute = exact_products(a, w, offsets, src)
    return c, want, product_error(absolute, Kd)


@pytest.mark.parametrize("counts,N,Kd", P_CASES)
def test_grouped_matmul_f32(counts, N, Kd):
    print("matmul f32", counts, N, Kd, flush=True)
    c, want, bound = run_matmul(counts, N, Kd, "f32", N + Kd, slack=5)
    c = c.double().cpu().numpy()
    assert (c[len(want):] == -7.0).all()                                   # rows behind the last group
    assert (np.abs(c[:len(want)] - want) <= bound + 1e-30).all(), np.max(np.abs(c[:len(want)] - want) / (bound + 1e-30))


# The matrix unit's 8-bit form cuts the eight products that it adds at once below 2^-13 of the largest one: at most
# 8 * 2^-13 of the sum of magnitudes, and in the 2-norm over many outputs far under bf16's rounding.
@pytest.mark.parametrize("counts,N,Kd", P_CASES)
@pytest.mark.parametrize("mapped", [0, 3])
def test_grouped_matmul_bf16(counts, N, Kd, mapped):
    print("matmul bf16", counts, N, Kd, mapped, flush=True)
    c, want, bound = run_matmul(counts, N, Kd, "bf16", N * 3 + Kd, slack=4, mapped=mapped)
    c = c.double().cpu().numpy()
    assert (c[len(want):] == -7.0).all()
    absolute = bound / product_error(1.0, Kd)
    err = np.abs(c[:len(want)] - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * 1.01 * absolute + bound).all()
    assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want)


def test_one_group_without_offsets():
    g = np.random.default_rng(5)
    rows, N, Kd = 70, 96, 288
    a, w = quantize(g.standard_normal((rows, Kd))), quantize(g.standard_normal((1, N, Kd)), BLOCK)
    outs = []
    for offsets in (None, tensor(np.array([0, rows], np.int32))):
        c = torch.full((rows, N), float("nan"), device="cuda")
        bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=rows, N=N, Kd=Kd, E=1, K=1, dtype=bm.BM_F32), tensor(a[0]), tensor(a[1]),
                             None, offsets, tensor(w[0]), tensor(w[1]), c)
        outs.append(c)
    assert torch.equal(*outs)
    want = values(*a) @ values(w[0][0], w[1][0], BLOCK).T
    np.testing.assert_allclose(outs[0].double().cpu().numpy(), want, atol=product_error(np.abs(values(*a)) @ np.abs(values(w[0][0], w[1][0], BLOCK)).T, Kd).max())


def test_256_groups_and_repeated_rows():
    """The largest number of groups, some of one row; the same token in several groups and several times in one."""
    print("256 groups", flush=True)
    g = np.random.default_rng(8)
    counts = g.integers(0, 4, 256)
    counts[[0, 63, 64, 255]] = [0, 2, 70, 3]
    offsets = grouped(counts, g)
    rows, N, Kd = int(offsets[-1]), 64, 64
    a, (w,) = inputs(counts, N, Kd, 9, a_rows=3)
    src = g.integers(0, 3, rows).astype(np.int32)
    c = torch.empty((rows, N), device="cuda")
    bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=3, N=N, Kd=Kd, E=256, K=1, dtype=bm.BM_F32), tensor(a[0]), tensor(a[1]), tensor(src),
                         tensor(offsets), tensor(w[0]), tensor(w[1]), c)
    want, absolute = exact_products(a, w, offsets, src)
    assert (np.abs(c.double().cpu().numpy() - want) <= product_error(absolute, Kd) + 1e-30).all()


def test_offsets_and_maps_that_leave_their_ranges():
    """Offsets past the rows, negative or falling, and mapped rows outside a: clamped.  Only that nothing outside c is written
    and that rows of well-formed groups are right is asked."""
    print("clamped offsets", flush=True)
    rows, N, Kd = 40, 64, 128
    g = np.random.default_rng(2)
    a, w = quantize(g.standard_normal((rows, Kd))), quantize(g.standard_normal((4, N, Kd)), BLOCK)
    room = torch.full((rows + 64, N), -7.0, device="cuda")
    c = room[32:32 + rows]
    offsets = np.array([-5, 10, 10, 30, 1 << 30], np.int32)                # groups 0..9, none, 10..29, 30..39
    src = np.arange(rows, dtype=np.int32)
    src[3], src[12] = -9, 1 << 30                                          # first and last row of a
    bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=rows, N=N, Kd=Kd, E=4, K=1, dtype=bm.BM_F32), tensor(a[0]), tensor(a[1]), tensor(src),
                         tensor(offsets), tensor(w[0]), tensor(w[1]), c)
    assert (room[:32] == -7.0).all() and (room[32 + rows:] == -7.0).all()
    src[3], src[12] = 0, rows - 1
    want, absolute = exact_products(a, w, np.array([0, 10, 10, 30, rows]), src)
    assert (np.abs(c.double().cpu().numpy() - want) <= product_error(absolute, Kd)).all()
    falling = np.array([30, 20, 40, 5, 0], np.int32)
    bm.bm_grouped_matmul(bm.ProductDesc(rows=rows, a_rows=rows, N=N, Kd=Kd, E=4, K=1, dtype=bm.BM_F32), tensor(a[0]), tensor(a[1]), None,
                         tensor(falling), tensor(w[0]), tensor(w[1]), c)
    torch.cuda.synchronize()
    assert (room[:32] == -7.0).all() and (room[32 + rows:] == -7.0).all()


def test_a_nan_stays_in_its_row_and_its_column():
    print("nan", flush=True)
    g = np.random.default_rng(4)
    counts, N, Kd = [20, 30], 96, 160
    a, (w,) = inputs(counts, N, Kd, 11)
    a[0][7, 130] = 0x7f                                                    # in the cut last block
    w[0][1, 5, 3] = 0xff
    offsets = grouped(counts, g)
    c = torch.empty((50, N), device="cuda")
    bm.bm_grouped_matmul(bm.ProductDesc(rows=50, a_rows=50, N=N, Kd=Kd, E=2, K=1, dtype=bm.BM_F32), tensor(a[0]), tensor(a[1]), None,
                         tensor(offsets), tensor(w[0]), tensor(w[1]), c)
    bad = np.zeros((50, N), bool)
    bad[7] = True
    bad[20:, 5] = True
    np.testing.assert_array_equal(np.isnan(c.cpu().numpy()), bad)


# ---- swiglu ----------------------------------------------------------------------------------------------------------


def check_swiglu(h, s, want_g, want_u, eg, eu, N):
    """h [rows][N] bytes and its scales against the exact gate and up products and the bounds of their errors."""
    hw = silu(want_g) * want_u
    # silu's slope is at most 1.1; exponential, reciprocal and products: eight roundings
    eh = 1.1 * np.abs(want_u) * eg + np.abs(silu(want_g)) * eu + 1.1 * eg * eu + 8 * 2.0 ** -24 * np.abs(hw)
    pad = [(0, 0), (0, -N % BLOCK)]
    blocks = lambda v: np.pad(v, pad).reshape(len(v), -1, BLOCK).max(2)   # noqa: E731
    want_s = np.maximum(blocks(np.abs(hw)) / 448, float(TINY))
    assert (np.abs(s - want_s) <= blocks(eh) / 448 + 2.0 ** -23 * want_s).all()
    S = spread(s.astype(np.float64), len(h), N, 1)
    err = np.abs(decode(h) * S - hw)
    assert (err <= np.maximum(2.0 ** -4 * (np.abs(hw) + eh), 2.0 ** -10 * S) * 1.001 + eh).all()


S_CASES = [([1], 32, 32, 1), ([3, 0, 2], 96, 64, 2), ([17, 1, 0, 64], 160, 128, 3), ([65, 0, 15], 256, 160, 1), ([33, 16], 768, 2048, 2),
           ([300, 0, 120], 352, 416, 2), ([129, 256, 257], 128, 256, 6), ([513, 140], 416, 1184, 1), ([1, 1, 1, 1], 1408, 4096, 8), ([130] * 9, 96, 224, 4)]


@pytest.mark.parametrize("counts,N,Kd,K", S_CASES)
def test_grouped_swiglu(counts, N, Kd, K):
    print("swiglu", counts, N, Kd, K, flush=True)
    g = np.random.default_rng(N + Kd)
    offsets = grouped(counts, g)
    rows, slack = int(offsets[-1]), 3
    T = -(-rows // K)
    a, (gate, up) = inputs(counts, N, Kd, N * 7 + Kd, T, matrices=2)
    perm = np.concatenate([g.permutation(T * K)[:rows], np.full(slack, -1)]).astype(np.int32)
    h = torch.full((rows + slack, N), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((rows + slack, -(-N // BLOCK)), -7.0, device="cuda")
    bm.bm_grouped_swiglu(bm.ProductDesc(rows=rows + slack, a_rows=T, N=N, Kd=Kd, E=len(counts), K=K), tensor(a[0]), tensor(a[1]), tensor(perm),
                         tensor(offsets), tensor(gate[0]), tensor(gate[1]), tensor(up[0]), tensor(up[1]), h, s)
    h, s = h.cpu().numpy(), s.cpu().numpy()
    assert (h[rows:] == 0x55).all() and (s[rows:] == -7.0).all()
    src = perm[:rows] // K
    wg, ag = exact_products(a, gate, offsets, src)
    wu, au = exact_products(a, up, offsets, src)
    check_swiglu(h[:rows], s[:rows], wg, wu, product_error(ag, Kd), product_error(au, Kd), N)
