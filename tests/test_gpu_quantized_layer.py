"""The layer on 8-bit experts: against numpy in 64 bits behind the oracle's routing, against its own operators one by one,
with every flag of the bf16 layer, in graphs and on streams (needs an MI355X)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2511_10054_amd as bm
import workloads
from helpers import HostLayer, to_device
from helpers_8bit import BLOCK, quantize, silu, tensor, values

pytestmark = pytest.mark.gpu


class Quantized:
    """A workload's layer with its experts in 8 bits; those of absent experts are NaN (nothing may read them)."""

    def __init__(self, name, over, T, base=None, flags=0, **gates):
        self.spec = workloads.scaled(name, **over)
        self.host = h = HostLayer(self.spec, T)
        s = self.spec
        if base is None:
            self.w = [quantize(h.f32(m), BLOCK) if m is not None else (None, None) for m in (h.wg, h.wu, h.wd, h.sg, h.su, h.sd)]
            for q, sc in self.w[:3]:
                q[~h.mask], sc[~h.mask] = 0x7f, np.nan
            self.dev = [tensor(t) if t is not None else None for m in self.w for t in m]
        else:
            self.w, self.dev = base.w, base.dev
        self.q = gates.pop("q", None)
        self.qd = tensor(self.q.astype(np.float32)) if self.q is not None else None
        self.gates = gates
        fl = bm.BM_RENORM_TOPK | flags
        fl |= (bm.BM_GATE_TAE if "tau" in gates else 0) | (bm.BM_GATE_MARGIN if "gamma" in gates else 0)
        fl |= (bm.BM_REPLACE_BUDGET if "rho" in gates else 0) | (bm.BM_GATE_DIST if "beta" in gates else 0) | (bm.BM_PSI_TOKEN if "eta" in gates else 0)
        self.desc = bm.LayerDesc(T=T, d=s.d, E=s.E, F=s.F, K=s.K, n_shared=s.n_shared, R=s.R, H=s.H, dtype=bm.BM_BF16, flags=fl,
                                 tae_tau=gates.get("tau", 0.0), margin_gamma=gates.get("gamma", 0.0), rho=gates.get("rho", 0),
                                 dist_beta=gates.get("beta", 0.0), psi_eta=gates.get("eta", 0.0))
        self.x, self.w_router, self.bias = to_device(h.x), to_device(h.w_router), to_device(h.bias)
        self.bitmap, self.table = to_device(h.bitmap), to_device(h.table)
        self.weights = bm.make_quantized_weights(self.w_router, self.bias, *self.dev, buddy_q=self.qd)
        self.work = torch.full((max(bm.bm_workspace_bytes_quantized(self.desc), 256),), 0xA5, dtype=torch.uint8, device="cuda")
        self.y = torch.full((T, s.d), float("nan"), dtype=torch.float32 if flags & bm.BM_Y_F32 else torch.bfloat16, device="cuda")

    def forward(self, x_q=None, x_scale=None, debug=True, stream=None):
        T, K, E = self.host.T, self.spec.K, self.spec.E
        i32 = dict(dtype=torch.int32, device="cuda")
        dbg = dict(ids=torch.full((T, K), -7, **i32), ids_remapped=torch.full((T, K), -7, **i32), w=torch.full((T, K), -7.0, device="cuda"),
                   offsets=torch.full((E + 1,), -7, **i32), perm=torch.full((T * K,), -7, **i32), inv_perm=torch.full((T * K,), -7, **i32),
                   stats=torch.full((6,), -7, **i32)) if debug else None
        bm.bm_moe_forward_quantized(self.desc, self.x, x_q, x_scale, self.weights, self.bitmap, self.table, self.y, self.work, dbg, stream)
        return dbg

    def reference(self, ids, w):
        """y in 64 bits for the ids after substitution and gate weights."""
        h = self.host
        x = values(*quantize(h.f32(h.x)))
        y = np.zeros((h.T, self.spec.d))

        def ffn(rows, mats, e):
            g, u = (rows @ values(m[0][e], m[1][e], BLOCK).T for m in mats[:2])
            return values(*quantize((silu(g) * u).astype(np.float32))) @ values(mats[2][0][e], mats[2][1][e], BLOCK).T

        for e in range(self.spec.E):
            t, k = np.nonzero(ids == e)
            if len(t):
                np.add.at(y, t, ffn(x[t], self.w[:3], e) * w[t, k][:, None])
        for e in range(self.spec.n_shared):
            y += ffn(x, self.w[3:], e)
        return y


# o and y in bf16 (half a step 2^-8 each, of the parts and of the whole, in the norm under both) and values of h that lie
# so near a border of e4m3 that the device's 32-bit sums put them on its other side: a sixteenth of few
LIMIT = 2.0 ** -7

LAYERS = [
    ("c4_qwen3", dict(d=256, F=96), 1, dict()),
    ("c4_qwen3", dict(d=256, F=256), 8, dict(flags=bm.BM_REMAP_UNIQUE, rho=1)),
    ("c2_mixtral_decode", dict(d=512, F=1024), 16, dict(flags=bm.BM_Y_F32)),
    ("c2_mixtral_decode", dict(d=512, F=1056), 64, dict()),
    ("c5_deepseek", dict(d=256, F=352), 33, dict(rho=1)),
    ("c5_deepseek", dict(d=288, F=1408), 300, dict(flags=bm.BM_REMAP_UNIQUE)),
    ("c3_mixtral_prefill", dict(d=384, F=512), 777, dict()),
    ("c4_qwen3", dict(d=256, F=160), 700, dict(flags=bm.BM_Y_F32)),
    ("c2_mixtral_decode", dict(d=256, F=512, n_resident=1), 40, dict()),
]


@pytest.mark.parametrize("name,over,T,kw", LAYERS)
def test_layer_matches_64_bits(name, over, T, kw):
    print("quantized layer", name, over, T, kw, flush=True)
    L = Quantized(name, over, T, **kw)
    out = {k: v.cpu().numpy() for k, v in L.forward().items()}
    y = L.y.double().cpu().numpy()
    ref = L.host.oracle_forward(oracle, unique=bool(kw.get("flags", 0) & bm.BM_REMAP_UNIQUE), rho=kw.get("rho"))
    np.testing.assert_array_equal(out["ids"], ref["ids"])
    np.testing.assert_array_equal(out["ids_remapped"], ref["ids_remapped"])
    want = L.reference(ref["ids_remapped"], ref["w"].astype(np.float64))
    rel = np.linalg.norm(y - want) / np.linalg.norm(want)
    print("   rel", rel, flush=True)
    assert np.isfinite(y).all() and rel <= LIMIT
    # and not far from the layer whose experts were not rounded to 8 bits
    assert np.linalg.norm(y - ref["y"]) <= 0.15 * np.linalg.norm(ref["y"])


@pytest.mark.parametrize("name,over,T,kw", [
    ("c4_qwen3", dict(d=256, F=128), 50, dict(tau=0.7)), ("c4_qwen3", dict(d=256, F=128), 50, dict(gamma=0.3, rho=2)),
    ("c4_qwen3", dict(d=256, F=128), 20, dict(beta=0.4)), ("c5_deepseek", dict(d=256, F=128), 90, dict(beta=1.5, flags=bm.BM_REMAP_UNIQUE)),
    ("c4_qwen3", dict(d=256, F=128), 40, dict(eta=2.0)), ("c4_qwen3", dict(d=256, F=128), 70, dict(eta=2.0, beta=1.5)),
])
def test_routing_is_the_bf16_layers(name, over, T, kw):
    """Every index array, the gate weights and the statistics are those of bm_moe_forward, whatever the gates."""
    print("routing", name, T, kw, flush=True)
    from helpers import DeviceLayer
    host = HostLayer(workloads.scaled(name, **over), T)
    if "eta" in kw:
        kw = dict(kw, q=np.random.default_rng(1).random((host.spec.E, host.spec.R)).astype(np.float32))
    want = DeviceLayer(host, unique=bool(kw.get("flags", 0)), **{k: v for k, v in kw.items() if k != "flags"}).forward()
    L = Quantized(name, over, T, **kw)
    out = L.forward()
    for k in ("ids", "ids_remapped", "w", "offsets", "perm", "inv_perm", "stats"):
        np.testing.assert_array_equal(out[k].cpu().numpy(), want[k], err_msg=k)
    assert torch.isfinite(L.y.float()).all()


@pytest.mark.parametrize("name,over,T", [("c5_deepseek", dict(d=256, F=352), 40), ("c2_mixtral_decode", dict(d=512, F=512), 300)])
def test_layer_is_the_chain_of_its_operators(name, over, T):
    """norm -> route -> substitute -> group -> swiglu -> matmul -> sum, each entry point called by the caller, against the
    layer on the norm's 8-bit output: the same routing, and y up to the sum's roundings."""
    print("chain", name, T, flush=True)
    L = Quantized(name, over, T)
    s = L.spec
    T, d, E, F, K = T, s.d, s.E, s.F, s.K
    g = torch.Generator(device="cuda").manual_seed(1)
    hidden, residual = L.x, torch.zeros_like(L.x)                          # a zero residual: the router's margins stay
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    xn, xr = torch.empty_like(L.x), torch.empty_like(L.x)
    xq, xs = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, -(-d // BLOCK)), device="cuda")
    bm.bm_add_rmsnorm(bm.NormDesc(T=T, d=d, dtype=bm.BM_BF16, eps=1e-6), hidden, residual, gamma, xr, xn, xq, xs)
    assert torch.equal(xr, hidden)
    L.x = xn
    dbg = L.forward(xq, xs)
    i32 = dict(dtype=torch.int32, device="cuda")
    ids, w, off, perm, inv = torch.empty((T, K), **i32), torch.empty((T, K), device="cuda"), torch.empty(E + 1, **i32), torch.empty(T * K, **i32), torch.empty(T * K, **i32)
    bm.bm_route_topk(L.desc, xn, L.w_router, L.bias, ids, w)
    bm.bm_buddy_remap(L.desc, L.bitmap, L.table, ids, ids, w)
    work = torch.empty(bm.bm_workspace_bytes(bm.LayerDesc(T=T, E=E, K=K)), dtype=torch.uint8, device="cuda")
    bm.bm_permute_by_expert(L.desc, ids, off, perm, inv, work)
    for k, v in dict(ids_remapped=ids, w=w, offsets=off, perm=perm, inv_perm=inv).items():
        assert torch.equal(dbg[k], v), k
    gq, gs, uq, us, dq, ds = L.dev[:6]
    h, hs = torch.empty((T * K, F), dtype=torch.uint8, device="cuda"), torch.empty((T * K, -(-F // BLOCK)), device="cuda")
    bm.bm_grouped_swiglu(bm.ProductDesc(rows=T * K, a_rows=T, N=F, Kd=d, E=E, K=K), xq, xs, perm, off, gq, gs, uq, us, h, hs)
    o = torch.zeros((T * K, d), dtype=torch.float32 if T <= 256 else torch.bfloat16, device="cuda")
    bm.bm_grouped_matmul(bm.ProductDesc(rows=T * K, a_rows=T * K, N=d, Kd=F, E=E, K=1, dtype=bm.BM_F32 if T <= 256 else bm.BM_BF16), h, hs, None, off, dq, ds, o)
    y = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    for k in range(K):
        at = inv.view(T, K)[:, k].long()
        y += torch.where((at >= 0)[:, None], o[at.clamp(min=0)].double() * w[:, k:k + 1].double(), 0.0)
    if s.n_shared:
        desc = bm.ProductDesc(rows=T, a_rows=T, N=F, Kd=d, E=1, K=1)
        for e in range(s.n_shared):
            m = [t[e:e + 1] for t in L.dev[6:]]
            hh, hhs = torch.empty((T, F), dtype=torch.uint8, device="cuda"), torch.empty((T, -(-F // BLOCK)), device="cuda")
            bm.bm_grouped_swiglu(desc, xq, xs, None, None, *m[:4], hh, hhs)
            oo = torch.empty((T, d), dtype=o.dtype, device="cuda")
            bm.bm_grouped_matmul(bm.ProductDesc(rows=T, a_rows=T, N=d, Kd=F, E=1, K=1, dtype=bm.BM_F32 if T <= 256 else bm.BM_BF16), hh, hhs, None, None, *m[4:], oo)
            y += oo.double()
    # K + n_shared additions in 32 bits and y's rounding; tiles of other heights may order a sum's blocks otherwise by nothing
    err, size = (L.y.double() - y).abs(), y.abs() + 2.0 ** -20 * y.abs().max()
    assert (err <= 2.0 ** -8 * 1.01 * size).all(), float((err / size).max())


def test_own_8_bit_tokens_are_bm_quantizes():
    L = Quantized("c4_qwen3", dict(d=256, F=128), 20)
    L.forward(debug=False)
    own = L.y.clone()
    q, s = torch.empty((20, 256), dtype=torch.uint8, device="cuda"), torch.empty((20, 2), device="cuda")
    bm.bm_quantize(bm.QuantizeDesc(n=1, rows=20, cols=256, block_rows=1, dtype=bm.BM_BF16), L.x, q, s)
    L.forward(q, s, debug=False)
    assert torch.equal(L.y, own)


@pytest.mark.parametrize("name,over,T,kw", [
    ("c4_qwen3", dict(d=256, F=64), 1, dict()), ("c5_deepseek", dict(d=96, F=64), 17, dict()), ("c2_mixtral_decode", dict(d=4096, F=32), 64, dict()),
    ("c4_qwen3", dict(d=160, F=32, E=256, n_resident=128), 40, dict()), ("c4_qwen3", dict(d=256, F=32), 2800, dict()),      # beside 16 | 8 waves, apart
    ("c4_qwen3", dict(d=288, F=32), 20, dict(beta=0.4)), ("c5_deepseek", dict(d=288, F=32), 90, dict(beta=0.4)),            # behind the batch's gate
])
def test_own_8_bit_tokens_at_every_front_end(name, over, T, kw):
    """Wherever the tokens' 8-bit form is made, y is what the tokens that bm_quantize makes give, call after call."""
    print("own tokens", name, over, T, kw, flush=True)
    L = Quantized(name, over, T, **kw)
    d = L.spec.d
    q, s = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, -(-d // BLOCK)), device="cuda")
    for turn in range(2):
        if turn:
            L.x.copy_(L.x.flip(0).clone() * 1.5)                           # other values in the same buffers
        L.forward(debug=False)
        own = L.y.clone()
        bm.bm_quantize(bm.QuantizeDesc(n=1, rows=T, cols=d, block_rows=1, dtype=bm.BM_BF16), L.x, q, s)
        L.work.fill_(0xA5)
        L.forward(q, s, debug=False)
        assert torch.equal(L.y, own) and torch.isfinite(own.float()).all()


@pytest.mark.parametrize("name,over,T,kw", [
    ("c4_qwen3", dict(d=256, F=256), 8, dict()), ("c5_deepseek", dict(d=256, F=352), 40, dict(rho=1)),
    ("c2_mixtral_decode", dict(d=512, F=512), 400, dict()), ("c4_qwen3", dict(d=256, F=128), 40, dict(beta=1.5))])
def test_replays_equal_eager(name, over, T, kw):
    """Captured once, replayed with new tokens in the same buffers and eager work in between."""
    print("graph", name, over, T, kw, flush=True)
    L = Quantized(name, over, T, **kw)
    xs = [to_device(HostLayer(L.spec, T, stream=i, base=L.host).x) for i in range(3)]
    eager = []
    for x in xs:
        L.x.copy_(x)
        L.forward(debug=False)
        eager.append(L.y.clone())
    assert not torch.equal(eager[0], eager[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.forward(debug=False)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.forward(debug=False)
    for rep in range(3):
        for i in (2, 0, 1):
            L.x.copy_(xs[i])
            L.y.zero_()
            L.work.fill_(0xFF)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(L.y, eager[i]), (rep, i)


def test_two_streams_with_workspaces_of_their_own():
    print("two streams", flush=True)
    A, B = Quantized("c4_qwen3", dict(d=256, F=256), 60), Quantized("c5_deepseek", dict(d=256, F=352), 400)
    want = []
    for L in (A, B):
        L.forward(debug=False)
        want.append(L.y.clone())
        L.y.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for L, st in ((A, streams[0]), (B, streams[1])):
            L.forward(debug=False, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(A.y, want[0]) and torch.equal(B.y, want[1])


def test_one_workspace_for_all_batches():
    print("kept workspace", flush=True)
    base = Quantized("c5_deepseek", dict(d=256, F=352), 300)
    for T in (300, 257, 256, 100, 1, 260):
        L = Quantized("c5_deepseek", dict(d=256, F=352), T, base=base)
        L.forward(debug=False)
        own = L.y.clone()
        L.work = base.work
        base.work.fill_(0xFF)
        L.forward(debug=False)
        assert torch.equal(L.y, own), T
    with pytest.raises(bm.BuddyMoEError):
        base.work = base.work[:-256]
        base.forward(debug=False)


def test_all_assignments_dropped():
    """No resident expert and no shared one: y is zero, no weight is read."""
    print("all dropped", flush=True)
    L = Quantized("c2_mixtral_decode", dict(d=256, F=256), 30)
    L.bitmap.zero_()
    dbg = L.forward()
    assert (dbg["ids_remapped"] == -1).all() and (L.y == 0).all()
