"""The layer on a routing that the caller has: bit for bit the layer that routes itself, and the whole way from the norm through
scored routing, 8-bit experts and a shared projection with adapters (needs an MI355X)."""
import numpy as np
import pytest

import workloads
from helpers import DeviceLayer, HostLayer, to_device
from helpers_8bit import BLOCK, quantize, tensor

pytestmark = pytest.mark.gpu

SHAPES = [
    ("c1_tiny", dict(), 16, dict(unique=True)),
    ("c1_tiny", dict(d=200, E=37, K=5), 77, dict(y_f32=True)),
    ("c2_mixtral_decode", dict(d=512, F=1024), 1, dict()),
    ("c2_mixtral_decode", dict(d=512, F=1024), 100, dict(unique=True)),
    ("c4_qwen3", dict(d=256, F=256), 8, dict(rho=1)),
    ("c4_qwen3", dict(d=256, F=256), 700, dict(unique=True, tau=0.9)),
    ("c5_deepseek", dict(d=256, F=1408), 40, dict(gamma=0.3)),
    ("c5_deepseek", dict(d=256, F=352), 600, dict(beta=0.5)),
    ("c5_deepseek", dict(d=256, F=352), 20, dict(beta=1.5)),
    ("c4_qwen3", dict(d=256, F=256), 5000, dict()),
]


def routed(dev, ids, w, y, **dbg):
    dev.bm.bm_moe_forward_routed(dev.desc, dev.x, ids, w, dev.weights, dev.bitmap, dev.table, y, dev.workspace, dbg or None)


@pytest.mark.parametrize("name,over,T,kw", SHAPES)
def test_same_bits_as_the_layer_that_routes(name, over, T, kw):
    import torch
    spec = workloads.scaled(name, **over)
    print("routed", name, over, T, kw, flush=True)
    dev = DeviceLayer(HostLayer(spec, T), **kw)
    bm = dev.bm
    ids, w = torch.empty((T, spec.K), dtype=torch.int32, device="cuda"), torch.empty((T, spec.K), device="cuda")
    bm.bm_route_topk(dev.desc, dev.x, dev.w_router, dev.bias, ids, w)
    want = dev.forward()
    given = ids.clone(), w.clone()
    A, E = T * spec.K, spec.E
    names = dict(ids=(A,), ids_remapped=(A,), offsets=(E + 1,), perm=(A,), inv_perm=(A,), stats=(6,))
    dbg = {k: torch.full(n, -9, dtype=torch.int32, device="cuda") for k, n in names.items()}
    dbg["w"] = torch.empty(A, device="cuda")
    y = torch.full_like(dev.y, float("nan"))
    weights = dev.weights
    no_router = bm.Weights.from_buffer_copy(weights)
    no_router.w_router = no_router.router_bias = None
    bm.bm_moe_forward_routed(dev.desc, dev.x, ids, w, no_router, dev.bitmap, dev.table, y, dev.workspace, dbg)
    torch.cuda.synchronize()
    assert torch.equal(ids, given[0]) and torch.equal(w, given[1])                 # inputs
    np.testing.assert_array_equal(y.float().cpu().numpy(), want["y"])
    for k in ("ids", "ids_remapped", "offsets", "perm", "inv_perm"):
        np.testing.assert_array_equal(dbg[k].cpu().numpy(), np.asarray(want[k]).reshape(-1), err_msg=k)
    np.testing.assert_array_equal(dbg["w"].cpu().numpy(), np.asarray(want["w"]).reshape(-1))
    np.testing.assert_array_equal(dbg["stats"].cpu().numpy(), np.asarray(want["stats"]))
    # without the intermediate arrays (whose counters then are not kept), and in a workspace that holds something else: the same bits
    for fill in (255, 1):
        dev.workspace.fill_(fill)
        y.fill_(float("nan"))
        bm.bm_moe_forward_routed(dev.desc, dev.x, ids, w, no_router, dev.bitmap, dev.table, y, dev.workspace)
        np.testing.assert_array_equal(y.float().cpu().numpy(), want["y"])


def test_ids_outside_and_ids_twice():
    """Slots without an expert count for nothing, an expert listed twice counts twice, whatever the weights' sum."""
    import torch
    spec = workloads.scaled("c1_tiny")
    dev = DeviceLayer(HostLayer(spec, 16, mask=np.ones(spec.E, bool)))
    one = torch.zeros((16, 2), dtype=torch.int32, device="cuda")
    w = torch.rand((16, 2), device="cuda") - 0.3
    ys = {}
    for key, ids, ww in (("twice", one, w), ("once", torch.stack([one[:, 0], one[:, 1] - 1], 1), torch.stack([w.sum(1), w[:, 0]], 1)),
                         ("far", torch.stack([one[:, 0], one[:, 1] + spec.E], 1), torch.stack([w.sum(1), w[:, 0]], 1)),
                         ("none", one - 5, w)):
        y = torch.empty_like(dev.y)
        routed(dev, ids.contiguous(), ww.contiguous(), y)
        ys[key] = y.double()
    assert torch.equal(ys["once"], ys["far"]) and (ys["none"] == 0).all()
    # the two halves are added after their products: three roundings of 2^-24 of at most |w0 o| + |w1 o|
    o = (ys["once"] / w.sum(1, keepdim=True)).abs()
    assert ((ys["twice"] - ys["once"]).abs() <= 5 * 2.0 ** -24 * o * w.abs().sum(1, keepdim=True)).all()


def small_model(seed, T=48, d=256, E=16, F=160, K=4, N=224):
    """Tensors of one block: norm, router, 8-bit experts with a shared one, a shared 8-bit projection and adapters."""
    import torch
    g = np.random.default_rng(seed)
    mask = np.ones(E, bool)
    mask[[2, 9, 11]] = False
    m = {"dims": (T, d, E, F, K, N), "mask": mask}
    for name, shape in (("gate", (E, F, d)), ("up", (E, F, d)), ("down", (E, d, F)), ("sgate", (1, F, d)), ("sup", (1, F, d)), ("sdown", (1, d, F)), ("proj", (1, N, d))):
        m[name] = [tensor(a) for a in quantize(g.standard_normal(shape).astype(np.float32) / np.sqrt(d), BLOCK)]
    m["table"] = tensor(np.stack([np.roll(np.arange(E), -i - 1)[:4] for i in range(E)]).astype(np.int32))
    m["bitmap"] = tensor(np.array([sum(1 << e for e in range(E) if mask[e])], np.int64))
    bf = lambda *s, f=1.0: torch.from_numpy((g.standard_normal(s) * f).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    m["x"], m["residual"], m["gamma"], m["router"] = bf(T, d), bf(T, d), bf(d, f=0.1) + 1, bf(E, d, f=d ** -0.5)
    m["balance"] = torch.from_numpy(g.standard_normal(E).astype(np.float32)).cuda() * 0.05
    m["a"], m["b"] = bf(3, 16, d, f=d ** -0.5), bf(3, N, 16, f=0.25)
    m["adapter"] = torch.from_numpy(g.integers(-1, 3, T).astype(np.int32)).cuda()
    m["scale"] = torch.tensor([0.5, 1.0, 2.0], device="cuda")
    return m


def run_block(bm, m, out):
    T, d, E, F, K, N = m["dims"]
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=1e-6), m["x"], m["residual"], m["gamma"], out["r"], out["n"], out["q"], out["s"])
    bm.bm_grouped_matmul(bm.ProductDesc(rows=T, a_rows=T, N=N, Kd=d, E=1, K=1, dtype=bm.BM_F32), out["q"], out["s"], None, None, *m["proj"], out["p"])
    ad = bm.AdapterDesc(rows=T, Kd=d, N=N, n=3, rank=16, dtype=bm.BM_BF16, y_dtype=bm.BM_F32)
    bm.bm_add_adapters(ad, out["n"], m["adapter"], m["a"], m["b"], None, m["scale"], out["p"], out["p"], out["wa"])
    rd = bm.RouterDesc(T=T, d=d, E=E, K=K, n_groups=4, keep_groups=2, group_top=2, scoring=bm.BM_SCORE_SIGMOID, dtype=bm.BM_BF16,
                       flags=bm.BM_RENORM_TOPK, scale=2.5)
    bm.bm_route_scored(rd, out["n"], m["router"], None, m["balance"], out["ids"], out["w"], out["wr"])
    ld = bm.LayerDesc(T=T, d=d, E=E, F=F, K=K, n_shared=1, R=4, H=4, dtype=bm.BM_BF16, flags=bm.BM_REMAP_UNIQUE | bm.BM_Y_F32)
    weights = bm.make_quantized_weights(None, None, *m["gate"], *m["up"], *m["down"], *m["sgate"], *m["sup"], *m["sdown"])
    bm.bm_moe_forward_routed_quantized(ld, None, out["q"], out["s"], out["ids"], out["w"], weights, m["bitmap"], m["table"], out["y"], out["wl"])


def outputs(bm, m):
    import torch
    T, d, E, F, K, N = m["dims"]
    e = lambda *s, t=torch.float32: torch.full(s, 7, dtype=t, device="cuda")  # noqa: E731
    return dict(r=e(T, d, t=torch.bfloat16), n=e(T, d, t=torch.bfloat16), q=e(T, d, t=torch.uint8), s=e(T, -(-d // 128)), p=e(T, N), ids=e(T, K, t=torch.int32),
                w=e(T, K), y=e(T, d), wa=e(8 << 20, t=torch.uint8), wr=e(1 << 20, t=torch.uint8), wl=e(16 << 20, t=torch.uint8))


def test_block_of_scored_routing_experts_and_adapters():
    """The operators one after the other, against their definitions in 64 bits on what the step before left; two captured graphs of
    two such blocks, each with workspaces of its own, replayed in turn."""
    import torch
    import paper_2511_10054_amd as bm
    from helpers_8bit import decode, silu, spread, values
    models = [small_model(s) for s in (3, 4)]
    outs = [outputs(bm, m) for m in models]
    for m, o in zip(models, outs):
        run_block(bm, m, o)
    torch.cuda.synchronize()
    m, o = models[0], {k: v.double().cpu().numpy() if v.dtype in (torch.float32, torch.bfloat16) else v.cpu().numpy() for k, v in outs[0].items() if k[0] != "w" or k == "w"}
    T, d, E, F, K, N = m["dims"]
    host = {k: [t.cpu().numpy() for t in m[k]] for k in ("gate", "up", "down", "sgate", "sup", "sdown", "proj")}
    x = values(o["q"], o["s"].astype(np.float32))
    # the projection with its adapters: fp32 sums of d and 16 products of values of order 1
    p = x @ values(host["proj"][0][0], host["proj"][1][0], BLOCK).T
    n, ad = o["n"], m["adapter"].cpu().numpy()
    for s in range(3):
        rows = ad == s
        p[rows] += float(m["scale"][s]) * (n[rows] @ m["a"][s].double().cpu().numpy().T) @ m["b"][s].double().cpu().numpy().T
    np.testing.assert_allclose(o["p"], p, atol=(d + 64) * 2.0 ** -24 * 4 * np.sqrt(d), rtol=0)
    # the routing on n; the layer on that routing
    z = n @ m["router"].double().cpu().numpy().T
    sc = 1 / (1 + np.exp(-z))
    for t in range(T):
        np.testing.assert_allclose(o["w"][t], 2.5 * sc[t, o["ids"][t]] / sc[t, o["ids"][t]].sum(), rtol=1e-4)
    y = np.zeros((T, d))
    mask, table = m["mask"], m["table"].cpu().numpy()

    def expert(names, e, row):
        gate, up, down = (values(host[k][0][e], host[k][1][e], BLOCK) for k in names)
        h = silu(row @ gate.T) * (row @ up.T)
        hq, hs = quantize(h[None].astype(np.float32))
        return values(hq, hs)[0] @ down.T

    for t in range(T):
        used = set(o["ids"][t].tolist())
        for k in range(K):
            e = int(o["ids"][t, k])
            if not mask[e]:
                e = next((int(b) for b in table[e] if mask[b] and int(b) not in used), -1)
                used.add(e)
            if e >= 0:
                y[t] += o["w"][t, k] * expert(("gate", "up", "down"), e, x[t])
        y[t] += expert(("sgate", "sup", "sdown"), 0, x[t])
    # h falls on another e4m3 value now and then where 32 bits and 64 differ: a step of 2^-4 of a few of 160 values
    assert np.linalg.norm(o["y"] - y) <= 2e-3 * np.linalg.norm(y)
    graphs, held = [], [{k: v.clone() for k, v in x.items()} for x in outs]
    for mm, oo in zip(models, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run_block(bm, mm, oo)
        graphs.append(graph)
    for rep in range(3):
        for i in (1, 0):
            for k, v in outs[i].items():
                v.fill_(3)
        for i in (0, 1):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            for k in ("r", "n", "q", "s", "p", "ids", "w", "y"):
                assert torch.equal(outs[i][k], held[i][k]), (rep, i, k)


@pytest.mark.parametrize("T,dist", [(1, False), (9, True), (300, False), (2500, True)])
def test_quantized_layer_same_bits_as_the_layer_that_routes(T, dist):
    import torch
    import paper_2511_10054_amd as bm
    m = small_model(5, T=T)
    _, d, E, F, K, N = m["dims"]
    flags = bm.BM_RENORM_TOPK | (bm.BM_GATE_DIST if dist else 0)
    ld = bm.LayerDesc(T=T, d=d, E=E, F=F, K=K, n_shared=1, R=4, H=4, dtype=bm.BM_BF16, flags=flags, dist_beta=0.9)
    args = [*m["gate"], *m["up"], *m["down"], *m["sgate"], *m["sup"], *m["sdown"]]
    work = torch.empty(bm.bm_workspace_bytes_quantized(ld), dtype=torch.uint8, device="cuda")
    ids, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    bm.bm_route_topk(ld, m["x"], m["router"], m["balance"], ids, w)
    ys = [torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    bm.bm_moe_forward_quantized(ld, m["x"], None, None, bm.make_quantized_weights(m["router"], m["balance"], *args), m["bitmap"], m["table"], ys[0], work)
    weights = bm.make_quantized_weights(None, None, *args)
    bm.bm_moe_forward_routed_quantized(ld, m["x"], None, None, ids, w, weights, m["bitmap"], m["table"], ys[1], work)
    q, s = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, d // 128), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=T, cols=d, block_rows=1, dtype=bm.BM_BF16), m["x"], q, s)
    bm.bm_moe_forward_routed_quantized(ld, None, q, s, ids, w, weights, m["bitmap"], m["table"], ys[2], work)
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
