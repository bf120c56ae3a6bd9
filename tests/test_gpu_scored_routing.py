"""Routing by scores, a balance bias and groups of experts against its definition in 64 bits (needs an MI355X).

Tokens and router weights are small multiples of powers of two, so that every logit is exact in 32 bits: what is compared is the
scores, the groups, the choice and the weights.  One case has logits that are not."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

INF = float("inf")


def reference(z, c, balance):
    """ids, weights, and which tokens no rounding of a score (2^-20 of it) turns: choices and group scores are told apart or equal."""
    T, E = z.shape
    G, per = c["G"], E // c["G"]
    with np.errstate(invalid="ignore", over="ignore"):
        if c["scoring"] == "softmax":
            s = np.exp(z - z.max(1, keepdims=True))
            s = s / s.sum(1, keepdims=True)
        else:
            s = 1.0 / (1.0 + np.exp(-z))
        v = s + (0.0 if balance is None else balance.astype(np.float64))
    v[np.isnan(v)] = -INF
    near = 2.0 ** -20 * np.where(np.isfinite(v), np.abs(v), 0).max(1) + 1e-300
    firm = np.ones(T, bool)

    def told_apart(a, keep):
        """The keep first of the falling a and the next are apart, or equal to the bit."""
        a = -np.sort(-a, axis=1)[:, : keep + 1]
        with np.errstate(invalid="ignore"):
            gap = a[:, :-1] - a[:, 1:]
        return ((gap > near[:, None]) | (a[:, :-1] == a[:, 1:]) | np.isnan(gap)).all(1)

    if c["keep"] < G:
        g = -np.sort(-v.reshape(T, G, per), axis=2)[:, :, : c["top"]]
        with np.errstate(invalid="ignore"):
            g = g.sum(2)
        g[np.isnan(g)] = -INF
        firm &= told_apart(g, c["keep"])
        out = np.argsort(-g, axis=1, kind="stable")[:, c["keep"]:]
        for t in range(T):
            for i in out[t]:
                v[t, i * per: (i + 1) * per] = -INF
    firm &= told_apart(v, c["K"])
    ids = np.argsort(-v, axis=1, kind="stable")[:, : c["K"]]
    live = np.take_along_axis(v, ids, 1) > -INF
    w = np.where(live, np.take_along_axis(s, ids, 1), 0.0)
    if c.get("renorm", True):
        w = w / np.maximum(w.sum(1, keepdims=True), 2.0 ** -126)
    return np.where(live, ids, -1), w * c.get("scale", 1.0), firm


def inputs(c, seed):
    """x [T][d], w [E][d] with exact logits of deviation about 1 (multiples of 2^-8 or finer), float32."""
    g = np.random.default_rng(seed)
    x = g.integers(-2, 3, (c["T"], c["d"])).astype(np.float32)
    shift = int(np.ceil(np.log2(3.7 * np.sqrt(c["d"]))))
    return x, g.integers(-4, 5, (c["E"], c["d"])).astype(np.float32) * np.float32(2.0 ** -shift)


def call(c, x, w, bias, balance, ids=None, weights=None, work=None):
    import torch
    import paper_2511_10054_amd as bm
    T = x.shape[0]
    desc = bm.RouterDesc(T=T, d=c["d"], E=c["E"], K=c["K"], n_groups=c["G"], keep_groups=c["keep"], group_top=c["top"],
                         scoring=bm.BM_SCORE_SIGMOID if c["scoring"] == "sigmoid" else bm.BM_SCORE_SOFTMAX,
                         dtype=bm.BM_F32 if c["dtype"] == "f32" else bm.BM_BF16, flags=bm.BM_RENORM_TOPK if c.get("renorm", True) else 0,
                         scale=c.get("scale", 1.0))
    ids = torch.full((T, c["K"]), -9, dtype=torch.int32, device="cuda") if ids is None else ids
    weights = torch.full((T, c["K"]), -9.0, device="cuda") if weights is None else weights
    work = torch.empty(max(bm.bm_workspace_bytes_scored(desc), 256), dtype=torch.uint8, device="cuda") if work is None else work
    bm.bm_route_scored(desc, x, w, bias, balance, ids, weights, work)
    return ids, weights


def tensors(c, *arrays):
    import torch
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    return [None if a is None else torch.from_numpy(a).cuda().to(dt if a.ndim == 2 else torch.float32) for a in arrays]


def case(T, d, E, K, G=1, keep=1, top=1, scoring="softmax", dtype="bf16", **kw):
    return dict(T=T, d=d, E=E, K=K, G=G, keep=keep, top=top, scoring=scoring, dtype=dtype, **kw)


CASES = [
    case(1, 32, 1, 1), case(1, 4096, 256, 8, 8, 4, 2, "sigmoid", scale=2.5), case(64, 2048, 64, 6, 8, 3, 1, renorm=False),
    case(17, 96, 256, 32, 4, 2, 2, "sigmoid"), case(33, 160, 128, 32, 64, 16, 1), case(50, 64, 60, 4, 5, 3, 2, "softmax", "f32"),
    case(130, 201, 37, 5, dtype="f32"), case(77, 3, 64, 8, 8, 8, 2, "sigmoid", "f32"), case(300, 1440, 200, 10, 8, 1, 2),
    case(1000, 512, 255, 16, 3, 2, 1, "sigmoid", scale=-1.5), case(2049, 1056, 256, 8, 8, 4, 2, "sigmoid"), case(4100, 544, 64, 6, 8, 3, 1),
    case(3000, 96, 8, 2), case(5000, 2048, 128, 8), case(1500, 1443, 60, 4, 5, 3, 2, dtype="f32"), case(1200, 2048, 129, 6, 3, 1, 2, dtype="f32"),
    case(16384 + 37, 64, 66, 3, 2, 1, 2, "sigmoid"),
    # groups of half a wave; every width and cut of the tiled product: ends of rows inside a line, fewer lines than parts, fp32 too
    case(70, 128, 256, 5, 2, 1, 2), case(70, 128, 64, 5, 2, 1, 2, "sigmoid"), case(200, 64, 192, 6, 8, 3, 2), case(8200, 96, 256, 8, 8, 4, 2, "sigmoid"),
    case(4200, 100, 20, 3, dtype="f32"), case(4200, 132, 250, 4, 5, 2, 2, "sigmoid", "f32"), case(900, 4128, 100, 4), case(300, 4160, 250, 4, 2, 1, 1), case(5000, 160, 30, 2),
    case(2100, 32, 64, 6, 8, 2, 2), case(700, 2052, 90, 4, dtype="f32"), case(5000, 999, 33, 2, dtype="f32"),
]


# Weights: a score is an exponential (2 units in the last place, and its argument rounded: up to 16 * 2^-24), a sum of E terms by 4 lane
# values and 6 exchanges, a quotient; then K additions, a quotient and a product: under 80 roundings of 2^-24.
W_TOL = 80 * 2.0 ** -24


@pytest.mark.parametrize("c", CASES, ids=lambda c: "T{T}-d{d}-E{E}-K{K}-G{G}x{keep}x{top}-{scoring}-{dtype}".format(**c))
@pytest.mark.parametrize("biased", ["none", "balance", "off"])
def test_choice_and_weights(c, biased):
    print("route", c, biased, flush=True)
    g = np.random.default_rng(7)
    x, w = inputs(c, c["T"] + c["d"])
    balance = bias = None
    if biased != "none":
        bias = g.integers(-8, 9, c["E"]).astype(np.float32) / 16
        balance = (g.standard_normal(c["E"]) * (0.1 if c["scoring"] == "sigmoid" else 0.3 / c["E"])).astype(np.float32)
    if biased == "off":
        balance[g.random(c["E"]) < 0.4] = -INF
    z = x.astype(np.float64) @ w.astype(np.float64).T + (0 if bias is None else bias)
    want_ids, want_w, firm = reference(z, c, balance)
    assert firm.mean() > 0.8
    ids, weights = call(c, *tensors(c, x, w, bias, balance))
    ids, weights = ids.cpu().numpy(), weights.double().cpu().numpy()
    np.testing.assert_array_equal(ids[firm], want_ids[firm])
    np.testing.assert_allclose(weights[firm], want_w[firm], rtol=W_TOL, atol=0)


@pytest.mark.parametrize("dtype,T,d", [("bf16", 700, 1024), ("f32", 300, 1000)])
def test_logits_that_round(dtype, T, d):
    """Weights of the choice against 64 bits: a logit is off by at most (d + 8) 2^-24 sum |x w|, and a token counts where twice that does
    not turn its choice."""
    import torch
    c = case(T, d, 96, 6, 8, 4, 2, "sigmoid", dtype)
    gen = torch.Generator(device="cuda").manual_seed(5)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w = torch.randn((T, d), generator=gen, device="cuda").to(dt), (torch.randn((96, d), generator=gen, device="cuda") / d ** 0.5).to(dt)
    ids, weights = (t.cpu().numpy() for t in call(c, x, w, None, None))
    xs, ws = x.double().cpu().numpy(), w.double().cpu().numpy()
    z, bound = xs @ ws.T, (d + 8) * 2.0 ** -24 * (np.abs(xs) @ np.abs(ws).T).max()
    want_ids, want_w, _ = reference(z, c, None)
    s = 1.0 / (1.0 + np.exp(-z))
    groups = -np.sort(-(-np.sort(-s.reshape(T, 8, 12), axis=2)[:, :, :2]).sum(2), axis=1)
    kept = s.copy()
    # (a sigmoid's slope is at most 1 / 4: choices move by bound / 4, group scores by bound / 2)
    firm = groups[:, 3] - groups[:, 4] > 1.01 * bound
    best = np.argsort(-(-np.sort(-s.reshape(T, 8, 12), axis=2)[:, :, :2]).sum(2), axis=1, kind="stable")[:, 4:]
    for t in range(T):
        for i in best[t]:
            kept[t, i * 12: (i + 1) * 12] = -1
    v = -np.sort(-kept, axis=1)[:, :7]
    firm &= ((v[:, :-1] - v[:, 1:]) > 0.51 * bound).all(1)
    print("firm", firm.mean(), "bound", bound, flush=True)
    assert firm.mean() > 0.3
    np.testing.assert_array_equal(ids[firm], want_ids[firm])
    np.testing.assert_allclose(weights[firm], want_w[firm], rtol=2 * bound + W_TOL)


@pytest.mark.parametrize("dtype,T,d,E", [("bf16", 4000, 1056, 256), ("bf16", 5000, 2048, 60), ("f32", 1100, 1000, 128), ("bf16", 17000, 96, 33)])
def test_a_tokens_bits_do_not_depend_on_its_batch(dtype, T, d, E):
    import torch
    c = case(T, d, E, 4, 1 if E == 33 else 4, 1 if E == 33 else 2, 2, "softmax", dtype)
    gen = torch.Generator(device="cuda").manual_seed(6)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w = torch.randn((T, d), generator=gen, device="cuda").to(dt), (torch.randn((E, d), generator=gen, device="cuda") / d ** 0.5).to(dt)
    ids, weights = call(c, x, w, None, None)
    again = call(c, x, w, None, None)
    assert torch.equal(ids, again[0]) and torch.equal(weights, again[1])
    for lo, n in ((0, 1), (5, 17), (T - 1, 1), (T // 2, 300), (T - 900, 900)):
        i, v = call(c, x[lo: lo + n].contiguous(), w, None, None)
        assert torch.equal(i, ids[lo: lo + n]) and torch.equal(v, weights[lo: lo + n]), (lo, n)


def test_equal_choices_go_to_the_lower_index():
    import torch
    for E, G, keep in ((64, 1, 1), (64, 8, 2), (256, 4, 3), (130, 2, 1)):
        c = case(5, 32, E, 7, G, keep, 1, "softmax")
        x, w = torch.zeros((5, 32), dtype=torch.bfloat16, device="cuda"), torch.ones((E, 32), dtype=torch.bfloat16, device="cuda")
        ids, weights = call(c, x, w, None, None)
        assert torch.equal(ids.cpu(), torch.arange(7, dtype=torch.int32).expand(5, 7)), (E, G)
        np.testing.assert_allclose(weights.cpu().numpy(), 1 / 7, rtol=W_TOL)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,keep", [(1, 1), (4, 2)])
def test_rows_and_experts_that_are_not_numbers(scoring, G, keep):
    """NaN and infinities stay in their rows; experts whose choice is NaN or -inf are never chosen; +inf comes first."""
    import torch
    c = case(6, 32, 40, 12, G, keep, 2, scoring)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn((6, 32), generator=gen, device="cuda").bfloat16(), torch.randn((40, 32), generator=gen, device="cuda").bfloat16()
    clean = call(c, x, w, None, None)
    x[2, 5] = float("nan")
    ids, weights = call(c, x, w, None, None)
    assert (ids[2] == -1).all() and (weights[2] == 0).all()
    rest = [0, 1, 3, 4, 5]
    assert torch.equal(ids[rest], clean[0][rest]) and torch.equal(weights[rest], clean[1][rest])
    # no expert is left
    ids, weights = call(c, x, w, None, torch.full((40,), -INF, device="cuda"))
    assert (ids == -1).all() and (weights == 0).all()
    # two experts are left, a NaN and an infinity among the balance
    b = torch.full((40,), -INF, device="cuda")
    b[3], b[7], b[8] = 0.0, INF, float("nan")
    ids, weights = call(c, x[:2].contiguous(), w, None, b)
    assert torch.equal(ids[:, :2].cpu(), torch.tensor([[7, 3]] * 2, dtype=torch.int32)) and (ids[:, 2:] == -1).all()
    np.testing.assert_allclose(weights.sum(1).cpu().numpy(), 1.0, rtol=W_TOL)
    # scores that vanish: weights are zeros, not NaN
    if scoring == "sigmoid":
        ids, weights = call(c, x[:2].contiguous(), w, torch.full((40,), -1000.0, device="cuda"), None)
        assert (ids >= 0).all() and (weights == 0).all()


def test_arrays_at_any_four_byte_address_and_rows_behind_the_last():
    import torch
    c = case(70, 100, 48, 5, 4, 2, 2, "sigmoid", "f32")
    gen = torch.Generator(device="cuda").manual_seed(2)
    store = torch.randn(70 * 100 + 48 * 100 + 8, generator=gen, device="cuda")
    x, w = store[1: 7001].view(70, 100), store[7003: 7003 + 4800].view(48, 100)
    bias = torch.randn(60, generator=gen, device="cuda")[3:51]
    want = call(c, x.clone(), w.clone(), bias.clone(), None)
    ids, weights = torch.full((73, 5), -9, dtype=torch.int32, device="cuda"), torch.full((73, 5), -9.0, device="cuda")
    call(c, x, w, bias, None, ids, weights)
    assert torch.equal(ids[:70], want[0]) and torch.equal(weights[:70], want[1])
    assert (ids[70:] == -9).all() and (weights[70:] == -9).all()


@pytest.mark.parametrize("T", [1, 40, 3000])
def test_graph_and_streams(T):
    """Captured once and replayed on new tokens with eager work in between, on a side stream too: the eager bits."""
    import torch
    c = case(T, 512, 128, 8, 8, 4, 2, "sigmoid")
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = (torch.randn((128, 512), generator=gen, device="cuda") / 22).bfloat16()
    xs = [torch.randn((T, 512), generator=gen, device="cuda").bfloat16() for _ in range(3)]
    want = [call(c, x, w, None, None) for x in xs]
    x = xs[0].clone()
    out = (torch.empty_like(want[0][0]), torch.empty_like(want[0][1]))
    work = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(c, x, w, None, None, *out, work)
    side.synchronize()
    assert torch.equal(out[0], want[0][0]) and torch.equal(out[1], want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c, x, w, None, None, *out, work)
    for _ in range(3):
        for i in (2, 0, 1):
            x.copy_(xs[i])
            out[0].fill_(-9)
            work.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[i][0]) and torch.equal(out[1], want[i][1])
