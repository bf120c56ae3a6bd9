"""Low-rank adapters of many requests beside a shared projection against their formula in 64 bits (needs an MI355X)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step, of the value


def case(rows, Kd, N, n, rank, dtype="bf16", y="bf16", order="any", none=0.2, ranks="own", scale=True, pad=(0, 0, 0), shift=0):
    return dict(rows=rows, Kd=Kd, N=N, n=n, rank=rank, dtype=dtype, y=y, order=order, none=none, ranks=ranks, scale=scale, pad=pad, shift=shift)


def make(c, seed=0):
    """Tensors of a case; what lies behind an adapter's own rank is NaN; rows of strided arrays stand in wider ones, at `shift` values."""
    import torch
    g = np.random.default_rng([seed, c["rows"], c["Kd"], c["N"], c["rank"]])
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    gen = torch.Generator(device="cuda").manual_seed(seed * 977 + c["rows"])

    def array(*shape, f=1.0, t="bf16"):
        return (f * torch.randn(shape, generator=gen, device="cuda")).to(dt[t])

    def placed(v, pad):
        store = torch.full((v.numel() + v.shape[0] * pad + c["shift"],), 5.0, dtype=v.dtype, device="cuda")
        at = store[c["shift"]:].view(v.shape[0], v.shape[1] + pad)[:, : v.shape[1]]
        at.copy_(v)
        return at, store

    n, r = c["n"], c["rank"]
    ids = g.integers(0, n, c["rows"])
    if c["order"] == "runs":
        ids = np.sort(ids)
    elif c["order"] == "one":
        ids[:] = n - 1
    ids = np.where(g.random(c["rows"]) < c["none"], g.choice([-1, -7, n, n + 500, 2 ** 31 - 1, -2 ** 31], c["rows"]), ids).astype(np.int32)
    ranks = g.integers(0, r + 1, n).astype(np.int32) if c["ranks"] == "own" else None
    s = dict(c=c, ids=ids, host_ranks=np.full(n, r) if ranks is None else ranks)
    s["adapter"] = torch.from_numpy(ids).cuda()
    s["ranks"] = None if ranks is None else torch.from_numpy(ranks).cuda()
    if ranks is not None and n > 2:                                        # clamped to [0, rank]
        ranks[:2] = r, 0
        s["ranks"] = torch.from_numpy(np.concatenate([[r + 3, -4], ranks[2:]]).astype(np.int32)).cuda()
    s["scale"] = (torch.rand(n, generator=gen, device="cuda") * 3 - 1) if c["scale"] else None
    s["x"], s["x_store"] = placed(array(c["rows"], c["Kd"], t=c["dtype"]), c["pad"][0])
    s["base"], s["base_store"] = placed(array(c["rows"], c["N"], t=c["y"]), c["pad"][1])
    s["y"], s["y_store"] = placed(array(c["rows"], c["N"], t=c["y"]) * float("nan"), c["pad"][2])
    a, b = array(n, r, c["Kd"], f=c["Kd"] ** -0.5, t=c["dtype"]), array(n, c["N"], r, f=r ** -0.5, t=c["dtype"])
    s["clean"] = a.clone(), b.clone()
    for i in range(n):
        a[i, s["host_ranks"][i]:] = float("nan")
        b[i, :, s["host_ranks"][i]:] = float("nan")
    s["a"], s["b"] = a, b
    if c["shift"]:
        s["a"], s["b"] = (torch.cat([torch.zeros(c["shift"], dtype=v.dtype, device="cuda"), v.flatten()])[c["shift"]:].view(v.shape) for v in (a, b))
    return s


def desc(c, in_place=False):
    import paper_2511_10054_amd as bm
    kinds = {"bf16": bm.BM_BF16, "f32": bm.BM_F32}
    strides = [w + p if p else 0 for w, p in zip((c["Kd"], c["N"], c["N"]), c["pad"])]
    if in_place:
        strides[2] = strides[1]
    return bm.AdapterDesc(rows=c["rows"], Kd=c["Kd"], N=c["N"], n=c["n"], rank=c["rank"], x_stride=strides[0], base_stride=strides[1], y_stride=strides[2],
                          dtype=kinds[c["dtype"]], y_dtype=kinds[c["y"]])


def call(s, in_place=False, work=None):
    import torch
    import paper_2511_10054_amd as bm
    d = desc(s["c"], in_place)
    work = torch.full((bm.bm_workspace_bytes_adapters(d),), 255, dtype=torch.uint8, device="cuda") if work is None else work
    bm.bm_add_adapters(d, s["x"], s["adapter"], s["a"], s["b"], s["ranks"], s["scale"], s["base"], s["base"] if in_place else s["y"], work)
    return s["base"] if in_place else s["y"]


def reference(s):
    """y and its bound.  u = A x: Kd products and additions in 32 bits, up to 16 parts and 4 waves; where B multiplies it, u is the sum of
    two bf16 values for a bf16 y (each off by half a step: 2^-16 of u), of three for an fp32 one (2^-24), or itself in fp32; B u: as many
    products of them, and zeros up to the next multiple of 32; then scale, addition (2^-24 each) and y's rounding."""
    c = s["c"]
    x, base = s["x"].double().cpu().numpy(), s["base"].double().cpu().numpy()
    a, b = (v.double().cpu().numpy() for v in s["clean"])
    scale = np.ones(c["n"]) if s["scale"] is None else s["scale"].double().cpu().numpy()
    y, bound = base.copy(), np.zeros_like(base)
    split = 2.0 ** -16 if c["dtype"] == "bf16" and c["y"] == "bf16" else 2.0 ** -24
    for i in range(c["n"]):
        rows, r = np.nonzero(s["ids"] == i)[0], int(s["host_ranks"][i])
        if not len(rows) or not r:
            continue
        u, ua = x[rows] @ a[i, :r].T, np.abs(x[rows]) @ np.abs(a[i, :r]).T
        du = (c["Kd"] + 24) * 2.0 ** -24 * ua + split * np.abs(u)
        mags = (np.abs(u) + du) @ np.abs(b[i, :, :r]).T
        d = scale[i] * (u @ b[i, :, :r].T)
        y[rows] += d
        bound[rows] = abs(scale[i]) * (du @ np.abs(b[i, :, :r]).T + (3 * r + 40) * 2.0 ** -24 * mags) + 2.0 ** -23 * (np.abs(base[rows]) + np.abs(d))
    live = bound > 0
    bound = np.where(live, bound + HALF[c["y"]] * (np.abs(y) + bound), 0.0)
    return y, bound


CASES = [
    case(1, 4096, 4096, 8, 16, none=0.0), case(1, 32, 64, 1, 1, ranks=None), case(2, 64, 16, 3, 8, y="f32"), case(5, 8, 8, 2, 8, ranks=None, scale=False),
    case(64, 256, 320, 32, 64), case(64, 512, 256, 64, 16, y="f32", order="runs"), case(63, 96, 72, 5, 128), case(65, 160, 257, 4, 128, y="f32", none=0.0),
    case(200, 1024, 1000, 3, 17, order="runs"), case(129, 100, 130, 4, 33, order="one", none=0.0), case(1023, 128, 96, 6, 16), case(1024, 64, 192, 2, 48, y="f32"),
    case(1025, 96, 64, 7, 20, order="runs"), case(3000, 256, 512, 1, 16, none=0.0), case(2500, 128, 264, 300, 8), case(1100, 64, 64, 1024, 16, y="f32"),
    case(4100, 320, 384, 5, 128, order="runs", none=0.0), case(33, 33, 35, 4, 5, dtype="f32", y="f32"), case(777, 1442, 333, 5, 12, "f32", "f32"),
    case(40, 512, 512, 6, 64, "f32", "bf16"), case(300, 128, 256, 3, 128, "f32", "f32", "runs"), case(1, 1, 1, 1, 1, "f32", "f32", none=0.0, ranks=None),
    case(1, 1, 1, 1, 1, none=0.0, ranks=None), case(90, 256, 256, 4, 32, pad=(64, 32, 96)), case(90, 256, 250, 4, 32, y="f32", pad=(3, 5, 1)),
    case(70, 128, 128, 4, 16, shift=1), case(70, 128, 96, 4, 40, "f32", "f32", shift=3, pad=(1, 2, 3)), case(50, 64, 64, 3, 16, none=1.0),
    case(7, 96, 300, 3, 12, "f32", "f32"), case(16, 128, 264, 5, 16, y="f32"), case(16, 192, 520, 40, 8, none=0.5), case(9, 64, 256, 2, 16, "f32", "bf16", "one"),
    case(60, 512, 256, 2, 48, order="one", none=0.0), case(64, 300, 256, 2, 128, "f32", "f32", "one"), case(17, 128, 128, 1, 16, none=0.0, pad=(8, 8, 8)),
    case(1200, 64, 128, 4, 16, y="f32", none=0.9), case(600, 2048, 128, 2, 64, order="runs", none=0.0), case(16, 16384, 48, 4, 16),
]


def ident(c):
    return "{rows}x{Kd}x{N}-n{n}-r{rank}-{dtype}-{y}-{order}-p{pad}-s{shift}".format(**c)


@pytest.mark.parametrize("c", CASES, ids=ident)
def test_against_the_formula(c):
    import torch
    print("adapters", c, flush=True)
    s = make(c)
    stores = {k: s[k].clone() for k in ("x_store", "base_store")}
    want, bound = reference(s)
    y = call(s)
    got = y.double().cpu().numpy()
    err = np.abs(got - want)
    assert (err <= bound).all(), (np.nanmax(err / np.maximum(bound, 1e-30)), np.argwhere(~(err <= bound))[:4])
    assert (got[bound == 0] == want[bound == 0]).all()                            # rows without an adapter, or with one of rank 0: base to the bit
    for k, v in stores.items():
        assert torch.equal(s[k], v)
    if c["pad"][2]:                                                              # between the rows of y
        assert (s["y_store"][c["shift"]:].view(c["rows"], -1)[:, c["N"]:] == 5).all()
    again = make(c)
    assert torch.equal(call(again), y)
    # in place: the same bits
    s2 = make(c)
    assert torch.equal(call(s2, in_place=True), y)
    if c["pad"][1]:
        assert (s2["base_store"][c["shift"]:].view(c["rows"], -1)[:, c["N"]:] == 5).all()


def test_rows_without_an_adapter_are_left_alone_in_place():
    """In place they are neither read nor written: NaN payloads stay."""
    import torch
    c = case(130, 64, 96, 3, 16, y="f32", none=0.5)
    s = make(c)
    none = torch.from_numpy((s["ids"] < 0) | (s["ids"] >= 3)).cuda()
    bits = s["base"].view(torch.int32)
    bits[none] = 0x7fc01234
    call(s, in_place=True)
    assert (bits[none] == 0x7fc01234).all() and torch.isfinite(s["base"][~none]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [10, 100])
def test_rows_that_are_not_numbers_stay_by_themselves(dtype, rows):
    import torch
    c = case(rows, 96, 64, 2, 16, dtype, "f32", "one", none=0.0, ranks=None)
    s = make(c)
    want = call(s).clone()
    s["x"][3, 7], s["x"][5, 9] = float("nan"), float("inf")
    s["base"][7] = float("-inf")
    got = call(s)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[[3, 5, 7]] = False
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[3]).all() and not torch.isfinite(got[5]).any() and (got[7] == float("-inf")).all()


def test_a_workspace_of_a_larger_batch_serves_smaller_ones():
    import torch
    import paper_2511_10054_amd as bm
    big = case(5000, 512, 128, 3, 16)
    work = torch.full((bm.bm_workspace_bytes_adapters(desc(big)),), 255, dtype=torch.uint8, device="cuda")
    for rows in (1, 15, 64, 700, 1024, 1025, 3000):
        c = dict(big, rows=rows)
        s = make(c)
        want, bound = reference(s)
        got = call(s, work=work).double().cpu().numpy()
        assert (np.abs(got - want) <= bound).all(), rows


def test_rows_past_32_bit_offsets():
    """A strided batch whose last rows lie beyond 2^31 values and 2^32 bytes."""
    import torch
    import paper_2511_10054_amd as bm
    rows, Kd, N, stride = 70, 64, 128, 1 << 25
    store = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    wide = store.view(rows, stride)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, base = torch.randn((rows, Kd), generator=gen, device="cuda").bfloat16(), torch.randn((rows, N), generator=gen, device="cuda").bfloat16()
    wide[:, :Kd], wide[:, 1024: 1024 + N] = x, base
    a, b = torch.randn((2, 8, Kd), generator=gen, device="cuda").bfloat16(), torch.randn((2, N, 8), generator=gen, device="cuda").bfloat16()
    adapter = torch.arange(rows, dtype=torch.int32, device="cuda") % 3 - 1
    ys = []
    for xx, bb, st in ((x, base.clone(), 0), (wide[:, :Kd], wide[:, 1024: 1024 + N], stride)):
        d = bm.AdapterDesc(rows=rows, Kd=Kd, N=N, n=2, rank=8, x_stride=st, base_stride=st, y_stride=st, dtype=bm.BM_BF16, y_dtype=bm.BM_BF16)
        work = torch.empty(bm.bm_workspace_bytes_adapters(d), dtype=torch.uint8, device="cuda")
        bm.bm_add_adapters(d, xx, adapter, a, b, None, None, bb, bb, work)
        ys.append(bb)
    assert torch.equal(ys[0], ys[1])


@pytest.mark.parametrize("c", [case(1, 512, 256, 4, 16, none=0.0), case(40, 512, 256, 4, 32), case(1500, 256, 320, 6, 16, y="f32")], ids=ident)
def test_graph_and_streams(c):
    """Captured once, replayed with other rows and other adapters in the same buffers, eager work between: the eager bits."""
    import torch
    import paper_2511_10054_amd as bm
    sets = [make(c, seed) for seed in (1, 2, 3)]
    for s in sets:                                                                # one set of adapters
        s["a"], s["b"], s["ranks"], s["scale"] = (sets[0][k] for k in ("a", "b", "ranks", "scale"))
    want = [call(s).clone() for s in sets]
    s = sets[0]
    given = [{k: t[k].clone() for k in ("x", "base", "adapter")} for t in sets]
    work = torch.full((bm.bm_workspace_bytes_adapters(desc(c)),), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(s, work=work)
    side.synchronize()
    assert torch.equal(s["y"], want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, work=work)
    for _ in range(3):
        for i in (2, 0, 1):
            for k, v in given[i].items():
                s[k].copy_(v)
            s["y"].fill_(3)
            work.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(s["y"], want[i]), i
