"""The library's 8-bit operators as cases that can be timed and checked: the way from a hidden state to a Mixture-of-Experts
layer whose expert weights are held in e4m3 with a scale for each block of 128.

A case is one of
  norm      bm_add_rmsnorm: the residual's addition, the root-mean-square norm, and the result in 16 (32) bits for the
            router and in 8 bits with a scale for each 128 values for the experts
  quantize  bm_quantize: weights (a scale for each 128 x 128 block) or activations (for each 128 values of a row)
  product   bm_grouped_matmul: rows grouped by expert, each group with its expert's 8-bit matrix
  swiglu    bm_grouped_swiglu: gathered tokens with the 8-bit gate and up matrices of their experts, silu(gate) * up out
            in 8 bits with scales
  layer     bm_moe_forward_quantized: the whole layer with buddy substitution, by way of the two before

Shapes are those of the layers in workloads.CONFIGS and, among the drawn ones, other widths that the library takes.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False          # False: the operators in elementary torch operations; True: the library's calls

# hidden size, experts, expert width, experts per token, resident, shared experts, Zipf exponent of the router bias
SHAPES = {
    "mixtral": dict(d=4096, E=8, F=14336, K=2, R=7, resident=5, shared=0, zipf=1.1),
    "qwen3": dict(d=2048, E=128, F=768, K=8, R=8, resident=64, shared=0, zipf=1.0),
    "deepseek": dict(d=2048, E=64, F=1408, K=6, R=8, resident=16, shared=2, zipf=1.0),
}
BLOCK = 128          # values that share a scale
MOST = 448.0         # largest e4m3 value
TINY = 2.0 ** -126   # smallest scale
EPS = 1e-6           # of the norm
MARGIN = 1e-3        # smallest gap of the K + 1 leading router logits: expert ids do not hang on the order of a sum
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _groups(shape, T, **kw):
    c = {k: v for k, v in SHAPES[shape].items() if k != "shared"}
    return dict(c, T=T, **kw)


def listed():
    m, q, d = SHAPES["mixtral"], SHAPES["qwen3"], SHAPES["deepseek"]
    return [
        # in front of the layer, one sequence's next token: nothing but the latency of a call
        dict(kind="norm", T=1, d=m["d"], dtype="bf16", name="norm_decode_T1"),
        # in front of the layer, a whole prompt
        dict(kind="norm", T=8192, d=d["d"], dtype="bf16", name="norm_prefill_T8192"),
        # loading time: the gate matrices of all resident experts
        dict(kind="quantize", n=d["resident"], rows=d["F"], cols=d["d"], block_rows=BLOCK, dtype="bf16", name="quantize_weights_deepseek"),
        # activations in 32 bits, a width whose last block is cut, an odd number of rows
        dict(kind="quantize", n=1, rows=4095, cols=1440, block_rows=1, dtype="f32", name="quantize_rows_4095x1440"),
        # down projection of a serving batch: the weights' bytes count
        dict(kind="product", N=m["d"], Kd=m["F"], out="bf16", **_groups("mixtral", 64), name="product_mixtral_decode_T64"),
        # a plain product: one group, ragged sizes, sums out in 32 bits
        dict(kind="product", N=2080, Kd=1440, out="f32", T=1000, E=1, K=1, R=0, resident=1, zipf=0.0, d=1440, F=2080, name="product_one_group_1000x2080x1440"),
        # down projection of a prompt with many small experts, groups from a few to some thousand rows
        dict(kind="product", N=q["d"], Kd=q["F"], out="bf16", **_groups("qwen3", 2048), name="product_qwen3_prefill_T2048"),
        # gate and up of a decode step with many small experts
        dict(kind="swiglu", **_groups("qwen3", 8), name="swiglu_qwen3_decode_T8"),
        # gate and up of a whole prompt, four large experts resident: the matrix units count
        dict(kind="swiglu", **dict(_groups("mixtral", 4096), resident=4), name="swiglu_mixtral_prefill_T4096"),
        # the layer for one sequence's next token
        dict(kind="layer", T=1, **m, name="layer_mixtral_decode_T1"),
        # the layer for a full serving batch
        dict(kind="layer", T=64, **m, name="layer_mixtral_decode_T64"),
        # the layer for a long prompt, with shared experts
        dict(kind="layer", T=8192, **d, name="layer_deepseek_prefill_T8192"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "quantize", "product", "product", "swiglu", "swiglu", "layer", "layer"])
    if kind == "norm":
        d = rng.choice([rng.randint(1, 700), 32 * rng.randint(1, 128), 2048, 4096])
        return dict(kind="norm", T=_log_int(rng, 1, 8192), d=d, dtype=rng.choice(["bf16", "f32"]))
    if kind == "quantize":
        block = rng.choice([1, BLOCK])
        return dict(kind="quantize", n=rng.randint(1, 16) if block > 1 else 1, rows=_log_int(rng, 1, 4096), cols=_log_int(rng, 1, 4096),
                    block_rows=block, dtype=rng.choice(["bf16", "f32"]))
    if rng.random() < 0.5:
        shape = rng.choice(["mixtral", "qwen3", "deepseek"])
        c = dict(SHAPES[shape])
        c["resident"] = rng.randint(c["resident"] // 2, c["E"])
        T = _log_int(rng, 1, 2048 if shape == "mixtral" else 8192)
    else:                                   # other widths: multiples of 32, whose last blocks of 128 are cut
        E = _log_int(rng, 1, 96)
        K = rng.randint(1, min(8, E))
        c = dict(d=32 * _log_int(rng, 2, 128), E=E, F=32 * _log_int(rng, 2, 128), K=K, R=min(rng.randint(4, 8), E - 1),
                 resident=rng.randint((E + 1) // 2, E), shared=rng.choice([0, 0, 1, 2]), zipf=rng.choice([0.0, 1.0]))
        T = _log_int(rng, 1, 4096)
    if kind == "layer":
        return dict(kind="layer", T=T, **c)
    c.pop("shared")
    if kind == "product":
        return dict(kind="product", T=T, N=c["d"], Kd=c["F"], out=rng.choice(["bf16", "f32"]), **c)
    return dict(kind="swiglu", T=T, **c)


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + stream)
    return g


def _tables(c, seed):
    """Router bias, residency mask, buddy table (numpy): every other expert by popularity resident, buddies by low-rank co-activation."""
    rng = np.random.default_rng([seed, 7])
    E, R = c["E"], c["R"]
    rank = rng.permutation(E) + 1
    bias = (-c["zipf"] * np.log(rank)).astype(np.float32)
    by_rank = np.argsort(rank)
    mask = np.zeros(E, dtype=bool)
    mask[np.concatenate([by_rank[0::2], by_rank[1::2]])[: c["resident"]]] = True
    u = rng.gamma(0.5, 1.0, size=(E, 8)) + 1e-9
    u /= np.linalg.norm(u, axis=1, keepdims=True)
    m = u @ u.T
    np.fill_diagonal(m, -np.inf)
    table = np.argsort(-m, axis=1, kind="stable")[:, :R].astype(np.int32)
    return bias, mask, table


def _substitutes(mask, table):
    """Per expert: itself where resident, else its first resident buddy, else -1 (numpy)."""
    E = len(mask)
    near = np.concatenate([np.arange(E, dtype=np.int32)[:, None], table], axis=1)
    there = mask[near]
    return np.where(there.any(1), near[np.arange(E), there.argmax(1)], -1)


def _grouping(c, seed):
    """What bm_permute_by_expert gives for a routed batch: offsets [E + 1], perm [T * K] (numpy), live rows."""
    bias, mask, table = _tables(c, seed)
    rng = np.random.default_rng([seed, 11])
    z = rng.standard_normal((c["T"], c["E"]), dtype=np.float32) + bias
    ids = _substitutes(mask, table)[np.argsort(-z, axis=1)[:, : c["K"]]].reshape(-1)
    live = np.nonzero(ids >= 0)[0]
    order = live[np.argsort(ids[live], kind="stable")]
    perm = np.full(ids.size, -1, np.int32)
    perm[: len(order)] = order
    offsets = np.concatenate([[0], np.cumsum(np.bincount(ids[live], minlength=c["E"]))]).astype(np.int32)
    return offsets, perm, mask


def _unit_rows(g, rows, cols):
    x = torch.randn((rows, cols), generator=g, device="cuda")
    return x / x.square().mean(1, keepdim=True).sqrt()


def _stored(x, block_rows):
    """x [..][rows][cols] in e4m3 and its scales, as a loader or the step before has left them."""
    rows, cols = x.shape[-2:]
    up = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % block_rows))
    up = up.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, block_rows))
    most = up.abs().amax((-1, -3), keepdim=True)
    # a quotient of two tensors: torch multiplies by the reciprocal where the divisor is a number, and a scale that is off in
    # its last bit sends the many 16-bit values that lie half way between two e4m3 ones to either side
    scale = (most / torch.full_like(most, MOST)).clamp(min=TINY)
    q = (up / scale).to(torch.float8_e4m3fn).flatten(-4, -3).flatten(-2, -1)[..., :rows, :cols]
    return q.contiguous(), scale.squeeze(-1).squeeze(-2).contiguous()


def _weights(c, seed, stream, n, mask, rows, cols):
    """n 8-bit matrices [rows][cols] and their scales; experts that are not resident hold zeros, which nothing reads."""
    g = _generator(seed, stream)
    q = torch.zeros((n, rows, cols), dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.ones((n, -(-rows // BLOCK), -(-cols // BLOCK)), device="cuda")
    for e in range(n):
        if mask is None or mask[e]:
            q[e], s[e] = _stored(torch.randn((rows, cols), generator=g, device="cuda") / math.sqrt(c["d"]), BLOCK)
    return q, s


def _tokens(c, seed, w_router, bias):
    """RMS-normalised tokens; one whose routing hangs on a rounding is drawn again."""
    g = _generator(seed, 1)
    kept, have = [], 0
    while have < c["T"]:
        x = _unit_rows(g, c["T"] + c["T"] // 4 + 16, c["d"]).to(torch.bfloat16)
        z = x.double() @ w_router.double().T + bias.double()
        top = torch.topk(z, min(c["K"] + 1, c["E"]), dim=1).values
        kept.append(x[((top[:, :-1] - top[:, 1:]) >= MARGIN).all(1)])
        have += len(kept[-1])
    return torch.cat(kept)[: c["T"]].contiguous()


def prepare(case, seed):
    c = case
    s = {"c": c}
    cuda = dict(device="cuda")
    bits8 = dict(dtype=torch.float8_e4m3fn, device="cuda")
    if c["kind"] == "norm":
        g, dt = _generator(seed, 1), TYPES[c["dtype"]]
        T, d = c["T"], c["d"]
        s["x"] = torch.randn((T, d), generator=g, **cuda).to(dt)                                # what the attention gave
        s["residual"] = (3.0 * torch.randn((T, d), generator=g, **cuda)).to(dt)
        s["gamma"] = (1.0 + 0.2 * torch.randn(d, generator=g, **cuda)).to(dt)
        s["out"] = dict(residual=torch.empty((T, d), dtype=dt, **cuda), y=torch.empty((T, d), dtype=dt, **cuda),
                        q=torch.empty((T, d), **bits8), scale=torch.empty((T, -(-d // BLOCK)), **cuda))
        return s
    if c["kind"] == "quantize":
        s["src"] = torch.randn((c["n"], c["rows"], c["cols"]), generator=_generator(seed, 1), **cuda).to(TYPES[c["dtype"]])
        s["out"] = dict(q=torch.empty((c["n"], c["rows"], c["cols"]), **bits8),
                        scale=torch.empty((c["n"], -(-c["rows"] // c["block_rows"]), -(-c["cols"] // BLOCK)), **cuda))
        return s
    T, K, E = c["T"], c["K"], c["E"]
    if c["kind"] == "layer":
        d, F, n = c["d"], c["F"], c["shared"]
        bias, mask, table = _tables(c, seed)
        s["bias"], s["mask"], s["table"] = torch.from_numpy(bias).cuda(), torch.from_numpy(mask).cuda(), torch.from_numpy(table).cuda()
        words = np.zeros((E + 63) // 64, dtype=np.uint64)
        np.bitwise_or.at(words, np.nonzero(mask)[0] // 64, np.uint64(1) << (np.nonzero(mask)[0] % 64).astype(np.uint64))
        s["bitmap"] = torch.from_numpy(words.view(np.int64)).cuda()
        s["w_router"] = (torch.randn((E, d), generator=_generator(seed, 2), **cuda) / math.sqrt(d)).to(torch.bfloat16)
        s["x"] = _tokens(c, seed, s["w_router"], s["bias"])
        s["gate"], s["up"] = _weights(c, seed, 10, E, mask, F, d), _weights(c, seed, 11, E, mask, F, d)
        s["down"] = _weights(c, seed, 12, E, mask, d, F)
        s["shared"] = [_weights(c, seed, 13, n, None, F, d), _weights(c, seed, 14, n, None, F, d), _weights(c, seed, 15, n, None, d, F)]
        s["live"] = torch.from_numpy(np.nonzero(mask)[0]).cuda()                                # resident experts
        s["y"] = torch.empty((T, d), dtype=torch.bfloat16, **cuda)
        return s
    offsets, perm, mask = _grouping(c, seed)
    s["offsets"], s["perm"] = torch.from_numpy(offsets).cuda(), torch.from_numpy(perm).cuda()
    s["live"] = torch.from_numpy(np.nonzero(mask)[0]).cuda()
    s["rows"], s["largest"] = int(offsets[-1]), int(np.diff(offsets).max())
    g = _generator(seed, 1)
    if c["kind"] == "product":
        s["a"] = _stored(_unit_rows(g, T * K, c["Kd"]), 1)
        s["w"] = _weights(c, seed, 10, E, mask, c["N"], c["Kd"])
        s["out"] = torch.zeros((T * K, c["N"]), dtype=TYPES[c["out"]], **cuda)                  # rows of dropped assignments stay
        return s
    s["a"] = _stored(_unit_rows(g, T, c["d"]), 1)
    s["gate"], s["up"] = _weights(c, seed, 10, E, mask, c["F"], c["d"]), _weights(c, seed, 11, E, mask, c["F"], c["d"])
    s["out"] = dict(h=torch.zeros((T * K, c["F"]), **bits8), scale=torch.zeros((T * K, -(-c["F"] // BLOCK)), **cuda))
    return s


# ---- the plain form --------------------------------------------------------------------------------------------------


def _plain_quantize(x, block_rows=1):
    return _stored(x, block_rows)


def _plain_values(qs, block_rows):
    """The 32-bit values that 8-bit ones and their scales stand for."""
    q, s = qs
    s = s.repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]
    return q.float() * (s.repeat_interleave(BLOCK, -2)[..., : q.shape[-2], :] if block_rows > 1 else s)


def _plain_norm(s):
    c, dt = s["c"], TYPES[s["c"]["dtype"]]
    r = s["x"].float() + s["residual"].float()
    n = r * torch.rsqrt(r.square().mean(1, keepdim=True) + EPS) * s["gamma"].float()
    q, scale = _plain_quantize(n)
    return dict(residual=r.to(dt), y=n.to(dt), q=q, scale=scale)


def _plain_pack(x, offsets, largest):
    """Rows in group order as [groups][largest][..] (zeros behind each group's end), and where each row went."""
    p = torch.arange(len(x), device=x.device)
    group = torch.searchsorted(offsets[1:].contiguous(), p.to(offsets.dtype), right=True)
    rank = p - offsets[group]
    packed = torch.zeros((len(offsets) - 1, largest, x.shape[1]), device=x.device)
    packed[group, rank] = x
    return packed, group, rank


def _plain_grouped(x, offsets, largest, w):
    """x [rows][Kd] in group order, w [groups][N][Kd]."""
    packed, group, rank = _plain_pack(x, offsets, largest)
    return torch.bmm(packed, w.transpose(1, 2).contiguous())[group, rank]


def _of_live(s, name):
    return _plain_values((s[name][0][s["live"]], s[name][1][s["live"]]), BLOCK)


def _plain_offsets(s):
    """The resident experts' offsets: the others' groups are empty."""
    return torch.cat([s["offsets"][s["live"]], s["offsets"][-1:]])


def _plain_product(s):
    x = _plain_values(s["a"], 1)[: s["rows"]]
    s["out"][: s["rows"]] = _plain_grouped(x, _plain_offsets(s), max(s["largest"], 1), _of_live(s, "w")).to(s["out"].dtype)
    return s["out"]


def _plain_silu(g):
    return g / (1.0 + torch.exp(-g))


def _plain_swiglu(s):
    x = _plain_values(s["a"], 1)[(s["perm"][: s["rows"]] // s["c"]["K"]).long()]
    at, n = _plain_offsets(s), max(s["largest"], 1)
    h = _plain_silu(_plain_grouped(x, at, n, _of_live(s, "gate"))) * _plain_grouped(x, at, n, _of_live(s, "up"))
    q, scale = _plain_quantize(h)
    s["out"]["h"][: s["rows"]], s["out"]["scale"][: s["rows"]] = q, scale
    return s["out"]


def _plain_layer(s):
    c = s["c"]
    T, K, E = c["T"], c["K"], c["E"]
    z = s["x"].double() @ s["w_router"].double().T + s["bias"].double()
    top, ids = torch.topk(z, K, dim=1)
    w = torch.softmax(top, dim=1).float()
    near = torch.cat([torch.arange(E, device=z.device)[:, None], s["table"].long()], dim=1)
    there = s["mask"][near]
    first = near.gather(1, there.int().argmax(1, keepdim=True))[:, 0]
    ids = torch.where(there.any(1), first, torch.full_like(first, -1))[ids]
    x = _plain_values(_plain_quantize(s["x"]), 1)
    flat = ids.flatten()
    at = torch.nonzero(flat >= 0)[:, 0]
    at = at[torch.argsort(flat[at], stable=True)]
    counts = torch.bincount(flat[at], minlength=E)[s["live"]]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    most = max(int(counts.max()), 1)
    h = _plain_silu(_plain_grouped(x[at // K], offsets, most, _of_live(s, "gate"))) * _plain_grouped(x[at // K], offsets, most, _of_live(s, "up"))
    o = _plain_grouped(_plain_values(_plain_quantize(h), 1), offsets, most, _of_live(s, "down"))
    y = torch.zeros((T * K, c["d"]), device=x.device)
    y[at] = o * w.flatten()[at][:, None]
    y = y.view(T, K, -1).sum(1)
    if c["shared"]:
        gate, up, down = (_plain_values(m, BLOCK).transpose(1, 2).contiguous() for m in s["shared"])
        xs = x.expand(c["shared"], -1, -1).contiguous()
        h = _plain_silu(torch.bmm(xs, gate)) * torch.bmm(xs, up)
        y = y + torch.bmm(_plain_values(_plain_quantize(h), 1), down).sum(0)
    return y.to(s["y"].dtype)


# ---- the library's calls ---------------------------------------------------------------------------------------------


def _plan(s):
    """What a program keeps beside its weights: descriptors and, for the layer, its workspace."""
    import paper_2511_10054_amd as bm
    c = s["c"]
    kinds = {"bf16": bm.BM_BF16, "f32": bm.BM_F32}
    if c["kind"] == "norm":
        s["desc"] = bm.NormDesc(T=c["T"], d=c["d"], dtype=kinds[c["dtype"]], eps=EPS)
    elif c["kind"] == "quantize":
        s["desc"] = bm.QuantizeDesc(n=c["n"], rows=c["rows"], cols=c["cols"], block_rows=c["block_rows"], dtype=kinds[c["dtype"]])
    elif c["kind"] == "product":
        s["desc"] = bm.ProductDesc(rows=c["T"] * c["K"], a_rows=c["T"] * c["K"], N=c["N"], Kd=c["Kd"], E=c["E"], K=1, dtype=kinds[c["out"]])
    elif c["kind"] == "swiglu":
        s["desc"] = bm.ProductDesc(rows=c["T"] * c["K"], a_rows=c["T"], N=c["F"], Kd=c["d"], E=c["E"], K=c["K"], dtype=bm.BM_BF16)
    else:
        s["desc"] = bm.LayerDesc(T=c["T"], d=c["d"], E=c["E"], F=c["F"], K=c["K"], n_shared=c["shared"], R=c["R"], H=c["R"],
                                 dtype=bm.BM_BF16, flags=bm.BM_RENORM_TOPK)
        shared = [t for m in s["shared"] for t in m] if c["shared"] else [None] * 6
        s["weights"] = bm.make_quantized_weights(s["w_router"], s["bias"], *s["gate"], *s["up"], *s["down"], *shared)
        s["work"] = torch.empty(bm.bm_workspace_bytes_quantized(s["desc"]), dtype=torch.uint8, device="cuda")
    s["bm"] = bm


def _own_run(s):
    if "bm" not in s:
        _plan(s)
    bm, kind, o = s["bm"], s["c"]["kind"], s.get("out")
    if kind == "norm":
        bm.bm_add_rmsnorm(s["desc"], s["x"], s["residual"], s["gamma"], o["residual"], o["y"], o["q"], o["scale"])
    elif kind == "quantize":
        bm.bm_quantize(s["desc"], s["src"], o["q"], o["scale"])
    elif kind == "product":
        bm.bm_grouped_matmul(s["desc"], *s["a"], None, s["offsets"], *s["w"], o)
    elif kind == "swiglu":
        bm.bm_grouped_swiglu(s["desc"], *s["a"], s["perm"], s["offsets"], *s["gate"], *s["up"], o["h"], o["scale"])
    else:
        bm.bm_moe_forward_quantized(s["desc"], s["x"], None, None, s["weights"], s["bitmap"], s["table"], s["y"], s["work"])
        return s["y"]
    return o


def run(s):
    if own:
        return _own_run(s)
    kind = s["c"]["kind"]
    if kind == "norm":
        return _plain_norm(s)
    if kind == "quantize":
        q, scale = _plain_quantize(s["src"], s["c"]["block_rows"])
        return dict(q=q, scale=scale)
    return {"product": _plain_product, "swiglu": _plain_swiglu, "layer": _plain_layer}[kind](s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    c = case
    up = lambda n: -(-n // BLOCK)  # noqa: E731
    if c["kind"] == "norm":
        T, d, esz = c["T"], c["d"], 2 if c["dtype"] == "bf16" else 4
        return dict(bytes=4 * T * d * esz + d * esz + T * d + T * up(d) * 4, flops=6.0 * T * d)
    if c["kind"] == "quantize":
        n, r, k, esz = c["n"], c["rows"], c["cols"], 2 if c["dtype"] == "bf16" else 4
        return dict(bytes=n * r * k * (esz + 1) + 4 * n * -(-r // c["block_rows"]) * up(k), flops=2.0 * n * r * k)
    T, K, E, d, F = c["T"], c["K"], c["E"], c["d"], c["F"]
    offsets = _grouping(c, 1)[0]
    rows, groups = int(offsets[-1]), int((np.diff(offsets) > 0).sum())
    matrix = lambda n, k: n * k + 4 * up(n) * up(k)  # noqa: E731
    if c["kind"] == "product":
        n, k = c["N"], c["Kd"]
        return dict(bytes=4 * (E + 1) + groups * matrix(n, k) + rows * (k + 4 * up(k) + n * (2 if c["out"] == "bf16" else 4)), flops=2.0 * rows * n * k)
    if c["kind"] == "swiglu":
        return dict(bytes=4 * (E + 1) + groups * 2 * matrix(F, d) + min(T, rows) * (d + 4 * up(d)) + rows * (4 + F + 4 * up(F)), flops=4.0 * rows * F * d)
    head = T * d * 2 + E * d * 2 + E * 4 + E * c["R"] * 4
    return dict(bytes=head + (groups + c["shared"]) * (2 * matrix(F, d) + matrix(d, F)) + T * d * 2,
                flops=2.0 * T * d * E + 6.0 * (rows + c["shared"] * T) * d * F)


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    """Values that come out in 8 bits are left unrounded here (value / scale); 8-bit values in the middle of the layer are
    rounded to e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6, halves to even; the operator's scale and the
    quotient in front of that rounding are 32-bit numbers by definition (16-bit values often lie half way)."""
    c = case
    s = prepare(case, seed)

    def blocks(x):
        scales = torch.stack([x[..., k: k + BLOCK].abs().amax(-1) for k in range(0, x.shape[-1], BLOCK)], -1)
        return (scales / torch.full_like(scales, MOST)).clamp(min=TINY)

    def spread(scale, width):
        return scale[..., torch.arange(width, device=scale.device) // BLOCK]

    def e4m3(x, scale):
        v = (x / scale).float().double()
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(v / step) * step * scale

    def matrix(qs, e):
        q, sc = qs[0][e].double(), qs[1][e].double()
        return q * spread(sc, q.shape[1])[torch.arange(q.shape[0], device=q.device) // BLOCK]

    def glu(x, gate, up):
        g = x @ gate.T
        return g * torch.sigmoid(g) * (x @ up.T)

    if c["kind"] == "norm":
        r = s["x"].double() + s["residual"].double()
        y = r / torch.sqrt((r * r).sum(1, keepdim=True) / c["d"] + EPS) * s["gamma"].double()
        scale = blocks(y)
        return dict(residual=r, y=y, q=y / spread(scale, c["d"]), scale=scale)
    if c["kind"] == "quantize":
        x = s["src"].double()
        by_row = blocks(x)
        if c["block_rows"] == 1:
            return dict(q=x / spread(by_row, c["cols"]), scale=by_row)
        scale = torch.stack([by_row[:, r: r + BLOCK].amax(1) for r in range(0, c["rows"], BLOCK)], 1)
        return dict(q=x / spread(scale, c["cols"])[:, torch.arange(c["rows"], device="cuda") // BLOCK], scale=scale)
    T, K = c["T"], c["K"]
    if c["kind"] == "layer":
        z = s["x"].double() @ s["w_router"].double().T + s["bias"].double()
        order = torch.argsort(z, dim=1, descending=True, stable=True)[:, :K]
        p = torch.exp(z - z.amax(1, keepdim=True)).gather(1, order)
        p = p / p.sum(1, keepdim=True)
        bias, mask, table = _tables(c, seed)
        lut = [e if mask[e] else next((int(b) for b in table[e] if mask[b]), -1) for e in range(c["E"])]
        ids = torch.tensor(lut, device="cuda")[order]
        x = s["x"].double()
        x = e4m3(x, spread(blocks(x).float().double(), c["d"]))
        y = torch.zeros((T, c["d"]), dtype=torch.float64, device="cuda")

        def ffn(rows, gate, up, down):
            h = glu(rows, gate, up)
            return e4m3(h, spread(blocks(h).float().double(), c["F"])) @ down.T

        for e in range(c["E"]):
            t, k = torch.nonzero(ids == e, as_tuple=True)
            if len(t):
                y.index_add_(0, t, ffn(x[t], matrix(s["gate"], e), matrix(s["up"], e), matrix(s["down"], e)) * p[t, k][:, None])
        for e in range(c["shared"]):
            y += ffn(x, *(matrix(m, e) for m in s["shared"]))
        return y
    offsets = s["offsets"].tolist()
    a = s["a"][0].double() * spread(s["a"][1].double(), s["a"][0].shape[1])
    width = c["N"] if c["kind"] == "product" else c["F"]
    out = torch.zeros((T * K, width), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo and c["kind"] == "product":
            out[lo:hi] = a[lo:hi] @ matrix(s["w"], e).T
        elif hi > lo:
            out[lo:hi] = glu(a[torch.div(s["perm"][lo:hi], K, rounding_mode="floor").long()], matrix(s["gate"], e), matrix(s["up"], e))
    if c["kind"] == "product":
        return out
    scale = blocks(out)
    scale[s["rows"]:] = 0.0
    return dict(h=out / spread(scale, width).clamp(min=TINY), scale=scale)
