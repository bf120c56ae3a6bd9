"""The layer on a given routing with more than 128 experts and many slots: every launch that substitutes and groups it, on routings that
another router may leave - empty slots, ids outside, experts listed twice - against the oracle, and bit for bit against the
layer that routes itself (needs an MI355X)."""
import numpy as np
import pytest

import oracle
import workloads
from helpers import DeviceLayer, HostLayer, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24           # half a step of fp32

# T, E, K, R, n_shared, gates: 64 tokens of 16 slots are the last batch of one launch, 17 slots the first beyond; 65 tokens: substitution
# first, then grouping in one workgroup or with the substitution's histograms; 4200 tokens of 256 experts: too many of those for every
# workgroup to add up
SHAPES = [
    (1, 256, 32, 32, 0, dict(unique=True)), (64, 256, 16, 32, 1, dict(unique=True, rho=3)), (64, 256, 16, 32, 0, dict()), (64, 256, 17, 32, 0, dict(unique=True)),
    (64, 129, 8, 4, 2, dict(unique=True, rho=1)), (65, 200, 6, 8, 0, dict(unique=True)), (65, 256, 16, 32, 0, dict(rho=2)), (63, 256, 9, 7, 0, dict(unique=True)),
    (700, 200, 6, 8, 1, dict(unique=True)), (130, 256, 32, 32, 0, dict(unique=True)), (300, 192, 1, 5, 0, dict(rho=0)), (700, 256, 8, 32, 0, dict(beta=0.2)),
    (30, 256, 8, 16, 0, dict(beta=0.9)), (4200, 256, 6, 8, 0, dict(unique=True)), (4200, 256, 1, 8, 0, dict()), (97, 256, 12, 0, 0, dict()),
]


def other_routing(g, T, E, K):
    """Ids [T][K] and weights: a token's experts are apart, but for a tenth of the slots empty, some outside, and some of the slot before."""
    ids = np.argsort(g.random((T, E)) * (1 + np.arange(E) % 7), axis=1)[:, :K].astype(np.int32)
    kind = g.random((T, K))
    ids[kind < 0.1] = -1
    ids[kind > 0.97] = g.choice([E, E + 77, 2 ** 31 - 1, -2 ** 31], (kind > 0.97).sum())
    if K > 1:
        twice = (kind > 0.9) & (kind <= 0.97)
        twice[:, 0] = False
        ids[twice] = np.roll(ids, 1, axis=1)[twice]
    return ids, (g.random((T, K)) * 2).astype(np.float32)


def reference(x, ids, w, gate, up, down, shared):
    """y in 64 bits and its bound: fp32 sums of d and F products (one rounding a term, and the tree's), the activation's exponential and quotient
    (6 roundings, and 2 |g| of the argument's), its slope of at most 1.1, a product each, and K + n_shared weighted additions."""
    T, d = x.shape
    F = gate.shape[1]
    y, bound, mags = (np.zeros((T, d)) for _ in range(3))

    def add(t, f, e, mats):
        a, b, c = (m[e].astype(np.float64) for m in mats)
        v = x[t].astype(np.float64)
        g, u, ga, ua = v @ a.T, v @ b.T, np.abs(v) @ np.abs(a).T, np.abs(v) @ np.abs(b).T
        s = g / (1 + np.exp(-g))
        h = s * u
        dh = 1.1 * (d + 8) * U * ga * (np.abs(u) + (d + 8) * U * ua) + np.abs(s) * (d + 8) * U * ua + (8 + 2 * np.abs(g)) * U * np.abs(h)
        o, oa = h @ c.T, (np.abs(h) + dh) @ np.abs(c).T
        np.add.at(y, t, f[:, None] * o)
        np.add.at(mags, t, np.abs(f)[:, None] * (np.abs(o) + oa * (F + 8) * U))
        np.add.at(bound, t, np.abs(f)[:, None] * (dh @ np.abs(c).T + (F + 8) * U * oa))

    for e in np.unique(ids[ids >= 0]):
        t, k = np.nonzero(ids == e)
        add(t, w[t, k].astype(np.float64), e, (gate, up, down))
    for s in range(0 if shared[0] is None else len(shared[0])):
        add(np.arange(T), np.ones(T), s, shared)
    return y, 1.01 * (bound + (ids.shape[1] + 6) * U * mags)


@pytest.mark.parametrize("T,E,K,R,n_shared,gates", SHAPES)
def test_against_the_oracle(T, E, K, R, n_shared, gates):
    import torch
    print("routed", T, E, K, R, n_shared, gates, flush=True)
    spec = workloads.scaled("c1_tiny", d=64, E=E, F=32, K=K, R=R, H=R, n_resident=E // 2, n_shared=n_shared)
    host = HostLayer(spec, T)
    dev = DeviceLayer(host, **gates)
    g = np.random.default_rng([T, E, K])
    ids, w = other_routing(g, T, E, K)
    want_ids, want_w, stats = oracle.buddy_remap_gated(ids, host.mask, host.table, w, H=R, **gates)
    offsets, perm, inv = oracle.permute(want_ids, E)
    A = T * K
    dbg = {k: torch.full((n,), -9, dtype=torch.int32, device="cuda") for k, n in dict(ids=A, ids_remapped=A, offsets=E + 1, perm=A, inv_perm=A, stats=6).items()}
    dbg["w"] = torch.empty(A, device="cuda")
    d_ids, d_w, y = to_device(ids), to_device(w), torch.full((T, 64), float("nan"), device="cuda")
    weights = dev.bm.Weights.from_buffer_copy(dev.weights)
    weights.w_router = weights.router_bias = None
    dev.workspace.fill_(255)
    dev.bm.bm_moe_forward_routed(dev.desc, dev.x, d_ids, d_w, weights, dev.bitmap, dev.table, y, dev.workspace, dbg)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(d_ids.cpu().numpy(), ids)
    np.testing.assert_array_equal(d_w.cpu().numpy(), w)
    for k, v in (("ids", ids), ("ids_remapped", want_ids), ("offsets", offsets), ("perm", perm), ("inv_perm", inv), ("w", want_w.astype(np.float32))):
        np.testing.assert_array_equal(dbg[k].cpu().numpy(), v.reshape(-1), err_msg=k)
    assert dbg["stats"].cpu().tolist() == [stats[k] for k in ("n_miss", "n_substituted", "n_dropped", "n_requested", "n_requested_offloaded", "bypassed")]
    want, bound = reference(host.x, want_ids, want_w, host.wg, host.wu, host.wd, (host.sg, host.su, host.sd))
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= bound).all(), np.nanmax(err / np.maximum(bound, 1e-300))
    again = torch.empty_like(y)
    dev.workspace.fill_(1)
    dev.bm.bm_moe_forward_routed(dev.desc, dev.x, d_ids, d_w, weights, dev.bitmap, dev.table, again, dev.workspace)
    assert torch.equal(again, y)


WIDE = [
    ("c4_qwen3", dict(d=64, F=64, E=256, K=16, R=32, H=32, n_resident=100), 64, dict(unique=True, tau=0.9)),
    ("c4_qwen3", dict(d=64, F=64, E=256, K=17, R=32, H=32, n_resident=100), 64, dict(unique=True, gamma=0.2)),
    ("c4_qwen3", dict(d=256, F=256, E=256, K=8, n_resident=128, n_shared=1), 1, dict(unique=True)),
    ("c4_qwen3", dict(d=256, F=256, E=256, K=8, n_resident=128), 33, dict(rho=2)),
    ("c4_qwen3", dict(d=64, F=96, E=200, K=6, n_resident=100), 65, dict(unique=True)),
    ("c4_qwen3", dict(d=64, F=96, E=200, K=6, n_resident=100), 700, dict(unique=True, rho=1)),
    ("c4_qwen3", dict(d=256, F=320, E=256, K=8, n_resident=128, n_shared=1), 900, dict(tau=0.95)),
    ("c4_qwen3", dict(d=64, F=64, E=256, K=8, n_resident=256), 4200, dict()),
    ("c4_qwen3", dict(d=64, F=64, E=256, K=8, n_resident=64), 4200, dict(unique=True, beta=0.99)),
]


@pytest.mark.parametrize("name,over,T,kw", WIDE)
def test_same_bits_as_the_layer_that_routes(name, over, T, kw):
    import torch
    print("routed", over, T, kw, flush=True)
    spec = workloads.scaled(name, **over)
    dev = DeviceLayer(HostLayer(spec, T), **kw)
    bm = dev.bm
    ids, w = torch.empty((T, spec.K), dtype=torch.int32, device="cuda"), torch.empty((T, spec.K), device="cuda")
    bm.bm_route_topk(dev.desc, dev.x, dev.w_router, dev.bias, ids, w)
    want = dev.forward()
    A = T * spec.K
    dbg = {k: torch.full((n,), -9, dtype=torch.int32, device="cuda") for k, n in dict(ids_remapped=A, offsets=spec.E + 1, perm=A, inv_perm=A, stats=6).items()}
    dbg["w"] = torch.empty(A, device="cuda")
    y = torch.full_like(dev.y, float("nan"))
    bm.bm_moe_forward_routed(dev.desc, dev.x, ids, w, dev.weights, dev.bitmap, dev.table, y, dev.workspace, dbg)
    torch.cuda.synchronize()
    for k, v in dbg.items():
        np.testing.assert_array_equal(v.cpu().numpy(), np.asarray(want[k]).reshape(-1), err_msg=k)
    np.testing.assert_array_equal(y.float().cpu().numpy(), want["y"])


@pytest.mark.parametrize("T,K", [(1, 8), (64, 16), (64, 17), (700, 8), (4200, 4)])
def test_quantized_layer_of_256_experts(T, K):
    """The same bits as the layer that routes itself; an emptied slot is one whose expert lies outside."""
    import torch
    import paper_2511_10054_amd as bm
    print("routed 8 bits", T, K, flush=True)
    E, d, F, R = 256, 128, 64, 8
    gen = torch.Generator(device="cuda").manual_seed(T + K)
    randn = lambda *s, f=1.0: f * torch.randn(s, generator=gen, device="cuda")  # noqa: E731

    def stored(rows, cols):
        q, s = torch.empty((E, rows, cols), dtype=torch.uint8, device="cuda"), torch.empty((E, -(-rows // 128), -(-cols // 128)), device="cuda")
        bm.bm_quantize(bm.QuantizeDesc(n=E, rows=rows, cols=cols, block_rows=128, dtype=bm.BM_BF16), randn(E, rows, cols, f=cols ** -0.5).bfloat16(), q, s)
        return q, s

    args = [*stored(F, d), *stored(F, d), *stored(d, F), None, None, None, None, None, None]
    x, router, bias = randn(T, d).bfloat16(), randn(E, d, f=d ** -0.5).bfloat16(), randn(E, f=0.5)
    mask = torch.rand(E, generator=gen, device="cuda") < 0.5
    bits = (mask.cpu().numpy().reshape(-1, 64).astype(np.uint64) << np.arange(64, dtype=np.uint64)).sum(1, dtype=np.uint64)
    bitmap = torch.from_numpy(bits.view(np.int64)).cuda()
    table = torch.stack([torch.roll(torch.arange(E), -i - 1)[:R] for i in range(E)]).int().cuda().contiguous()
    ld = bm.LayerDesc(T=T, d=d, E=E, F=F, K=K, R=R, H=R, dtype=bm.BM_BF16, flags=bm.BM_RENORM_TOPK | bm.BM_REMAP_UNIQUE | bm.BM_Y_F32)
    work = torch.empty(bm.bm_workspace_bytes_quantized(ld), dtype=torch.uint8, device="cuda")
    ids, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    bm.bm_route_topk(ld, x, router, bias, ids, w)
    ys = [torch.full((T, d), float("nan"), device="cuda") for _ in range(4)]
    bm.bm_moe_forward_quantized(ld, x, None, None, bm.make_quantized_weights(router, bias, *args), bitmap, table, ys[0], work)
    weights = bm.make_quantized_weights(None, None, *args)
    bm.bm_moe_forward_routed_quantized(ld, x, None, None, ids, w, weights, bitmap, table, ys[1], work)
    assert torch.isfinite(ys[0]).all() and torch.equal(ys[0], ys[1])
    # the last slot emptied, in two ways
    for y, fill in ((ys[2], -1), (ys[3], E + 9)):
        none = ids.clone()
        none[:, -1] = fill
        bm.bm_moe_forward_routed_quantized(ld, x, None, None, none, w, weights, bitmap, table, y, work)
    assert torch.isfinite(ys[2]).all() and torch.equal(ys[2], ys[3]) and not torch.equal(ys[2], ys[1])
