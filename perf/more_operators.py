"""Operators around the Mixture-of-Experts layer as cases that can be timed and checked: routing by other scores than the plain
softmax, the layer behind such a router, and the low-rank adapters of many requests beside a shared projection.

A case is one of
  route     bm_route_scored: softmax or sigmoid scores, a bias for balance that only the choice sees, groups of experts, top-k,
            weights renormalised and scaled
  layer     bm_moe_forward_routed and bm_moe_forward_routed_quantized: the layer on expert ids and gate weights that are given
  adapters  bm_add_adapters: y = base + scale * B (A x), every row with the adapter of its request, or with none

Layers have the shapes of workloads.CONFIGS; the other sizes are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False          # False: the operators in elementary torch operations; True: the library's calls

# hidden size, experts, expert width, experts per token, buddy-table width, resident and shared experts, Zipf exponent of the popularity
SHAPES = {
    "mixtral": dict(d=4096, E=8, F=14336, K=2, R=7, resident=5, shared=0, zipf=1.1),
    "qwen3": dict(d=2048, E=128, F=768, K=8, R=8, resident=64, shared=0, zipf=1.0),
    "deepseek": dict(d=2048, E=64, F=1408, K=6, R=8, resident=16, shared=2, zipf=1.0),
}
BLOCK = 128          # values that share a scale (8-bit experts)
MOST = 448.0         # largest e4m3 value
TINY = 2.0 ** -126   # smallest normal number: of a scale, and of the sum that weights are divided by
MARGIN = 5e-5        # smallest gap of leading choices, of the largest one: expert ids do not hang on the order of a sum
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _route(T, d, E, K, groups=1, keep=1, top=1, scoring="softmax", dtype="bf16", renorm=True, scale=1.0, balance=True, off=0, **kw):
    return dict(kind="route", T=T, d=d, E=E, K=K, groups=groups, keep=keep, top=top, scoring=scoring, dtype=dtype, renorm=renorm, scale=scale,
                balance=balance, off=off, **kw)


def _adapters(T, Kd, N, n, rank, dtype="bf16", y="bf16", order="runs", none=0.0, mixed=False, **kw):
    return dict(kind="adapters", T=T, Kd=Kd, N=N, n=n, rank=rank, dtype=dtype, y=y, order=order, none=none, mixed=mixed, **kw)


def listed():
    q, d = SHAPES["qwen3"], SHAPES["deepseek"]
    return [
        # one sequence's next token, many experts in groups: latency
        _route(1, 4096, 256, 8, 8, 4, 2, "sigmoid", scale=2.5, name="route_sigmoid_groups_T1"),
        # a serving batch, groups scored by their best expert, plain softmax weights
        _route(64, 2048, 64, 6, 8, 3, 1, "softmax", renorm=False, balance=False, name="route_softmax_groups_T64"),
        # 32-bit router of an odd number of experts in five groups, ragged batch, some experts switched off
        _route(1000, 1440, 60, 4, 5, 3, 2, "softmax", "f32", off=2, name="route_f32_60_experts_T1000"),
        # a whole prompt, many experts in groups
        _route(8192, 4096, 256, 8, 8, 4, 2, "sigmoid", scale=2.5, name="route_sigmoid_groups_T8192"),
        # the layer behind another router: a decode batch with shared experts
        dict(kind="layer", T=32, experts="bf16", **d, name="layer_deepseek_decode_T32"),
        # the same of a prompt on 8-bit experts, many small ones
        dict(kind="layer", T=2048, experts="q8", **q, name="layer_qwen3_8bit_prefill_T2048"),
        # one sequence's next token with its adapter: latency
        _adapters(1, 4096, 4096, 8, 16, name="adapters_T1_rank16"),
        # a serving batch, requests of 32 adapters in any order, some without one
        _adapters(64, 4096, 4096, 32, 64, order="any", none=0.1, mixed=True, name="adapters_decode_T64_rank64"),
        # prompts of a few requests one after the other
        _adapters(8192, 2048, 4096, 6, 16, name="adapters_prompts_T8192_rank16"),
        # prompts and decode rows together, a large rank, the sums of an fp32 projection
        _adapters(2000, 4096, 1408, 24, 128, y="f32", order="tail", none=0.05, mixed=True, name="adapters_ragged_T2000_rank128"),
        # 32-bit adapters of odd sizes
        _adapters(777, 1442, 1001, 5, 12, "f32", "f32", order="any", none=0.2, name="adapters_f32_odd_T777"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["route", "route", "adapters", "adapters", "layer"])
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 5, 8])
        per = rng.randint(1 if groups > 1 else 2, 256 // groups)
        keep = rng.randint(1, groups)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = 32 * _log_int(rng, 1, 128) if dtype == "bf16" else _log_int(rng, 17, 2048)
        return _route(_log_int(rng, 1, 8192 if dtype == "bf16" else 2048), d, groups * per, rng.randint(1, min(16, keep * per)), groups, keep,
                      rng.randint(1, min(2, per)), rng.choice(["softmax", "sigmoid"]), dtype, rng.random() < 0.7, rng.choice([1.0, 2.5]),
                      rng.random() < 0.7, rng.randint(0, (per - 2) // 2) if per >= 4 and rng.random() < 0.3 else 0)
    if kind == "adapters":
        rank = rng.choice([8, 16, 32, 64, 128, rng.randint(1, 100)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        n = _log_int(rng, 1, max(1, min(64, 2048 // rank)))
        even = 32 if rng.random() < 0.5 else 1
        T = _log_int(rng, 1, 8192 if dtype == "bf16" else 2048)
        return _adapters(T, even * _log_int(rng, max(1, 33 // even), 4096 // even), even * _log_int(rng, max(1, 33 // even), 4096 // even), n, rank, dtype,
                         rng.choice(["bf16", "f32"]), rng.choice(["runs", "any", "tail"]), rng.choice([0.0, 0.1, 0.5]), rng.random() < 0.5)
    if rng.random() < 0.5:
        c = dict(SHAPES[rng.choice(["qwen3", "deepseek"])])
        c["resident"] = rng.randint(c["resident"] // 2, c["E"])
    else:
        E = _log_int(rng, 2, 96)
        c = dict(d=32 * _log_int(rng, 2, 64), E=E, F=32 * _log_int(rng, 2, 64), K=rng.randint(1, min(8, E)), R=min(rng.randint(4, 8), E - 1),
                 resident=rng.randint((E + 1) // 2, E), shared=rng.choice([0, 0, 1, 2]), zipf=rng.choice([0.0, 1.0]))
    return dict(kind="layer", T=_log_int(rng, 1, 2048), experts=rng.choice(["bf16", "q8"]), **c)


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + stream)
    return g


def _unit_rows(g, rows, cols):
    x = torch.randn((rows, cols), generator=g, device="cuda")
    return x / x.square().mean(1, keepdim=True).sqrt()


def _balance(c, seed):
    """What a trainer left to even out the experts' load; -inf switches an expert off (numpy, or None)."""
    if not c["balance"] and not c["off"]:
        return None
    rng = np.random.default_rng([seed, 21])
    b = rng.standard_normal(c["E"]) * (0.05 if c["scoring"] == "sigmoid" else 0.2 / c["E"]) * c["balance"]
    per = c["E"] // c["groups"]
    for g in range(c["groups"]):
        b[g * per + rng.permutation(per)[: c["off"]]] = -np.inf
    return b.astype(np.float32)


def _firm(c, z, balance):
    """Tokens whose choice no rounding turns: groups and experts are told apart by a margin."""
    s = torch.softmax(z, 1) if c["scoring"] == "softmax" else torch.sigmoid(z)
    v = s if balance is None else s + balance
    least = MARGIN * torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v)).amax(1)
    firm = torch.ones(len(z), dtype=torch.bool, device=z.device)
    if c["keep"] < c["groups"]:
        score = torch.topk(v.unflatten(1, (c["groups"], -1)), c["top"], dim=2).values.sum(2)
        top, at = torch.topk(score, c["keep"] + 1, dim=1)
        firm &= ~((top[:, -2] - top[:, -1]) < least)
        kept = torch.zeros_like(score, dtype=torch.bool).scatter(1, at[:, :-1], True)
        v = torch.where(kept.repeat_interleave(c["E"] // c["groups"], 1), v, torch.full_like(v, -math.inf))
    top = torch.topk(v, min(c["K"] + 1, c["E"]), dim=1).values
    return firm & ~((top[:, :-1] - top[:, 1:]) < least[:, None]).any(1)


def _tokens(c, seed, w_router, bias, balance):
    g = _generator(seed, 1)
    kept, have = [], 0
    while have < c["T"]:
        x = _unit_rows(g, c["T"] + c["T"] // 4 + 16, c["d"]).to(TYPES[c["dtype"]])
        kept.append(x[_firm(c, x.double() @ w_router.double().T + bias.double(), None if balance is None else balance.double())])
        have += len(kept[-1])
    return torch.cat(kept)[: c["T"]].contiguous()


def _requests(c, seed):
    """The adapter of every row, -1 for none (numpy): runs of prompts, any order, or prompts with decode rows behind them."""
    rng = np.random.default_rng([seed, 31])
    T, n = c["T"], c["n"]

    def runs(rows):
        cuts = np.sort(rng.integers(0, rows + 1, n - 1)) if rows else np.zeros(n - 1, np.int64)
        return np.repeat(rng.permutation(n), np.diff(np.concatenate([[0], cuts, [rows]])))

    if c["order"] == "runs":
        ids = runs(T)
    elif c["order"] == "any":
        ids = rng.integers(0, n, T)
    else:
        ids = np.concatenate([runs(T - T // 8), rng.integers(0, n, T // 8)])
    none = rng.random(T) < c["none"]
    ranks = rng.integers(1, c["rank"] + 1, n) if c["mixed"] else np.full(n, c["rank"])
    return np.where(none, -1, ids).astype(np.int32), ranks.astype(np.int32)


def _tables(c, seed):
    """Popularity of the experts, residency mask, buddy table (numpy): every other expert by popularity resident, buddies by
    low-rank co-activation."""
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
    return bias, mask, np.argsort(-m, axis=1, kind="stable")[:, :R].astype(np.int32)


def _routed(c, seed):
    """Expert ids [T][K] and gate weights as another router leaves them (numpy)."""
    bias = _tables(c, seed)[0]
    rng = np.random.default_rng([seed, 11])
    z = rng.standard_normal((c["T"], c["E"]), dtype=np.float32) + bias
    ids = np.argsort(-z, axis=1)[:, : c["K"]]
    w = 1.0 / (1.0 + np.exp(-np.take_along_axis(z, ids, 1)))
    return ids.astype(np.int32), (2.5 * w / w.sum(1, keepdims=True)).astype(np.float32)


def _substitutes(mask, table):
    """Per expert: itself where resident, else its first resident buddy, else -1 (numpy)."""
    E = len(mask)
    near = np.concatenate([np.arange(E, dtype=np.int32)[:, None], table], axis=1)
    there = mask[near]
    return np.where(there.any(1), near[np.arange(E), there.argmax(1)], -1)


def _stored(x, block_rows):
    """x [..][rows][cols] in e4m3 and its scales."""
    rows, cols = x.shape[-2:]
    up = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % block_rows))
    up = up.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, block_rows))
    most = up.abs().amax((-1, -3), keepdim=True)
    # a quotient of two tensors: torch multiplies by the reciprocal where the divisor is a number
    scale = (most / torch.full_like(most, MOST)).clamp(min=TINY)
    q = (up / scale).to(torch.float8_e4m3fn).flatten(-4, -3).flatten(-2, -1)[..., :rows, :cols]
    return q.contiguous(), scale.squeeze(-1).squeeze(-2).contiguous()


def _weights(c, seed, stream, n, mask, rows, cols):
    """n matrices [rows][cols], in bf16 or in 8 bits with scales; experts that are not resident hold zeros, which nothing reads."""
    g = _generator(seed, stream)
    q8 = c["experts"] == "q8"
    q = torch.zeros((n, rows, cols), dtype=torch.float8_e4m3fn if q8 else torch.bfloat16, device="cuda")
    s = torch.ones((n, -(-rows // BLOCK), -(-cols // BLOCK)), device="cuda") if q8 else None
    for e in range(n):
        if mask is None or mask[e]:
            m = torch.randn((rows, cols), generator=g, device="cuda") / math.sqrt(c["d"])
            if q8:
                q[e], s[e] = _stored(m, BLOCK)
            else:
                q[e] = m
    return q, s


def prepare(case, seed):
    c = case
    s = {"c": c}
    cuda = dict(device="cuda")
    T = c["T"]
    if c["kind"] == "route":
        dt = TYPES[c["dtype"]]
        s["w_router"] = (torch.randn((c["E"], c["d"]), generator=_generator(seed, 2), **cuda) / math.sqrt(c["d"])).to(dt)
        s["bias"] = 0.2 * torch.randn(c["E"], generator=_generator(seed, 3), **cuda)
        b = _balance(c, seed)
        s["balance"] = None if b is None else torch.from_numpy(b).cuda()
        s["x"] = _tokens(c, seed, s["w_router"], s["bias"], s["balance"])
        s["ids"] = torch.empty((T, c["K"]), dtype=torch.int32, **cuda)
        s["w"] = torch.empty((T, c["K"]), **cuda)
        return s
    if c["kind"] == "adapters":
        dt, yt, n, r = TYPES[c["dtype"]], TYPES[c["y"]], c["n"], c["rank"]
        ids, ranks = _requests(c, seed)
        s["adapter"], s["ranks"] = torch.from_numpy(ids).cuda(), torch.from_numpy(ranks).cuda()
        s["x"] = _unit_rows(_generator(seed, 1), T, c["Kd"]).to(dt)
        s["a"] = (torch.randn((n, r, c["Kd"]), generator=_generator(seed, 2), **cuda) / math.sqrt(c["Kd"])).to(dt)
        s["b"] = (torch.randn((n, c["N"], r), generator=_generator(seed, 3), **cuda) / math.sqrt(r)).to(dt)
        s["scale"] = 0.5 + torch.rand(n, generator=_generator(seed, 4), **cuda)
        s["base"] = torch.randn((T, c["N"]), generator=_generator(seed, 5), **cuda).to(yt)     # the shared projection's output
        s["y"] = torch.empty((T, c["N"]), dtype=yt, **cuda)
        return s
    E, d, F, n = c["E"], c["d"], c["F"], c["shared"]
    _, mask, table = _tables(c, seed)
    ids, w = _routed(c, seed)
    s["ids"], s["w"] = torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda()
    s["mask"], s["table"] = torch.from_numpy(mask).cuda(), torch.from_numpy(table).cuda()
    words = np.zeros((E + 63) // 64, dtype=np.uint64)
    np.bitwise_or.at(words, np.nonzero(mask)[0] // 64, np.uint64(1) << (np.nonzero(mask)[0] % 64).astype(np.uint64))
    s["bitmap"] = torch.from_numpy(words.view(np.int64)).cuda()
    s["x"] = _unit_rows(_generator(seed, 1), T, d).to(torch.bfloat16)
    s["gate"], s["up"] = _weights(c, seed, 10, E, mask, F, d), _weights(c, seed, 11, E, mask, F, d)
    s["down"] = _weights(c, seed, 12, E, mask, d, F)
    s["shared"] = [_weights(c, seed, 13, n, None, F, d), _weights(c, seed, 14, n, None, F, d), _weights(c, seed, 15, n, None, d, F)]
    s["live"] = torch.from_numpy(np.nonzero(mask)[0]).cuda()                                    # resident experts
    s["y"] = torch.empty((T, d), dtype=torch.bfloat16, **cuda)
    return s


# ---- the plain form --------------------------------------------------------------------------------------------------


def _plain_route(s):
    c = s["c"]
    z = s["x"].float() @ s["w_router"].float().T + s["bias"]
    if c["scoring"] == "softmax":
        p = torch.exp(z - z.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-z))
    v = p if s["balance"] is None else p + s["balance"]
    per = c["E"] // c["groups"]
    if c["keep"] < c["groups"]:
        score = torch.topk(v.view(-1, c["groups"], per), c["top"], dim=2).values.sum(2)
        kept = torch.zeros_like(score).scatter(1, torch.topk(score, c["keep"], dim=1).indices, 1.0) > 0
        v = torch.where(kept[:, :, None], v.view(-1, c["groups"], per), -math.inf).view(-1, c["E"])
    top, ids = torch.topk(v, c["K"], dim=1)
    live = top > -math.inf
    w = torch.where(live, p.gather(1, ids), 0.0)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=TINY)
    return dict(ids=torch.where(live, ids, -1).int(), w=w * c["scale"])


def _plain_adapters(s):
    """Every row with every adapter's A; of the products only those of its own adapter and within its rank stay."""
    c = s["c"]
    n, r = c["n"], c["rank"]
    u = (s["x"].float() @ s["a"].float().view(n * r, -1).T).view(-1, n, r)
    mine = (s["adapter"][:, None] == torch.arange(n, device=u.device))[:, :, None] & (torch.arange(r, device=u.device) < s["ranks"][:, None])
    u = torch.where(mine, u * s["scale"][:, None], 0.0).view(-1, n * r)
    return (s["base"].float() + u @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1)).to(s["y"].dtype)


def _plain_values(qs, block_rows):
    """The 32-bit values that a matrix stands for."""
    q, s = qs
    if s is None:
        return q.float()
    s = s.repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]
    return q.float() * (s.repeat_interleave(BLOCK, -2)[..., : q.shape[-2], :] if block_rows > 1 else s)


def _plain_of_live(s, name):
    q, sc = s[name]
    return _plain_values((q[s["live"]], None if sc is None else sc[s["live"]]), BLOCK)


def _plain_grouped(x, offsets, largest, w):
    """x [rows][Kd] in group order, w [groups][N][Kd]."""
    p = torch.arange(len(x), device=x.device)
    group = torch.searchsorted(offsets[1:].contiguous(), p, right=True)
    rank = p - offsets[group]
    packed = torch.zeros((len(offsets) - 1, largest, x.shape[1]), device=x.device)
    packed[group, rank] = x
    return torch.bmm(packed, w.transpose(1, 2).contiguous())[group, rank]


def _plain_silu(g):
    return g / (1.0 + torch.exp(-g))


def _plain_layer(s):
    c = s["c"]
    T, K, E = c["T"], c["K"], c["E"]
    q8 = c["experts"] == "q8"
    held = (lambda v: _plain_values(_stored(v, 1), 1)) if q8 else (lambda v: v.float())
    near = torch.cat([torch.arange(E, device=s["x"].device)[:, None], s["table"].long()], dim=1)
    there = s["mask"][near]
    first = near.gather(1, there.int().argmax(1, keepdim=True))[:, 0]
    flat = torch.where(there.any(1), first, torch.full_like(first, -1))[s["ids"].long()].flatten()
    x = held(s["x"])
    at = torch.nonzero(flat >= 0)[:, 0]
    at = at[torch.argsort(flat[at], stable=True)]
    counts = torch.bincount(flat[at], minlength=E)[s["live"]]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    most = max(int(counts.max()), 1)
    h = _plain_silu(_plain_grouped(x[at // K], offsets, most, _plain_of_live(s, "gate"))) * _plain_grouped(x[at // K], offsets, most, _plain_of_live(s, "up"))
    o = _plain_grouped(held(h), offsets, most, _plain_of_live(s, "down"))
    y = torch.zeros((T * K, c["d"]), device=x.device)
    y[at] = o * s["w"].flatten()[at][:, None]
    y = y.view(T, K, -1).sum(1)
    if c["shared"]:
        gate, up, down = (_plain_values(m, BLOCK).transpose(1, 2).contiguous() for m in s["shared"])
        xs = x.expand(c["shared"], -1, -1).contiguous()
        y = y + torch.bmm(held(_plain_silu(torch.bmm(xs, gate)) * torch.bmm(xs, up)), down).sum(0)
    return y.to(s["y"].dtype)


# ---- the library's calls ---------------------------------------------------------------------------------------------


def _plan(s):
    """What a program keeps beside its weights: descriptors and workspaces."""
    import paper_2511_10054_amd as bm
    c = s["c"]
    kinds = {"bf16": bm.BM_BF16, "f32": bm.BM_F32}
    if c["kind"] == "route":
        s["desc"] = bm.RouterDesc(T=c["T"], d=c["d"], E=c["E"], K=c["K"], n_groups=c["groups"], keep_groups=c["keep"], group_top=c["top"],
                                  scoring=bm.BM_SCORE_SIGMOID if c["scoring"] == "sigmoid" else bm.BM_SCORE_SOFTMAX, dtype=kinds[c["dtype"]],
                                  flags=bm.BM_RENORM_TOPK if c["renorm"] else 0, scale=c["scale"])
        need = bm.bm_workspace_bytes_scored(s["desc"])
    elif c["kind"] == "adapters":
        s["desc"] = bm.AdapterDesc(rows=c["T"], Kd=c["Kd"], N=c["N"], n=c["n"], rank=c["rank"], dtype=kinds[c["dtype"]], y_dtype=kinds[c["y"]])
        need = bm.bm_workspace_bytes_adapters(s["desc"])
    else:
        s["desc"] = bm.LayerDesc(T=c["T"], d=c["d"], E=c["E"], F=c["F"], K=c["K"], n_shared=c["shared"], R=c["R"], H=c["R"], dtype=bm.BM_BF16)
        m = [s["gate"], s["up"], s["down"]] + (s["shared"] if c["shared"] else [(None, None)] * 3)
        if c["experts"] == "q8":
            s["weights"] = bm.make_quantized_weights(None, None, *[t for qs in m for t in qs])
            need = bm.bm_workspace_bytes_quantized(s["desc"])
        else:
            s["weights"] = bm.make_weights(None, None, *[qs[0] for qs in m])
            need = bm.bm_workspace_bytes(s["desc"])
    s["work"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    s["bm"] = bm


def _own_run(s):
    if "bm" not in s:
        _plan(s)
    bm, kind = s["bm"], s["c"]["kind"]
    if kind == "route":
        bm.bm_route_scored(s["desc"], s["x"], s["w_router"], s["bias"], s["balance"], s["ids"], s["w"], s["work"])
        return dict(ids=s["ids"], w=s["w"])
    if kind == "adapters":
        bm.bm_add_adapters(s["desc"], s["x"], s["adapter"], s["a"], s["b"], s["ranks"], s["scale"], s["base"], s["y"], s["work"])
    elif s["c"]["experts"] == "q8":
        bm.bm_moe_forward_routed_quantized(s["desc"], s["x"], None, None, s["ids"], s["w"], s["weights"], s["bitmap"], s["table"], s["y"], s["work"])
    else:
        bm.bm_moe_forward_routed(s["desc"], s["x"], s["ids"], s["w"], s["weights"], s["bitmap"], s["table"], s["y"], s["work"])
    return s["y"]


def run(s):
    if own:
        return _own_run(s)
    return {"route": _plain_route, "adapters": _plain_adapters, "layer": _plain_layer}[s["c"]["kind"]](s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    c = case
    T = c["T"]
    if c["kind"] == "route":
        esz = 2 if c["dtype"] == "bf16" else 4
        return dict(bytes=(T + c["E"]) * c["d"] * esz + 4 * c["E"] * (1 + (c["balance"] or c["off"] > 0)) + 8 * T * c["K"], flops=2.0 * T * c["E"] * c["d"])
    if c["kind"] == "adapters":
        esz, ysz = (2 if c[k] == "bf16" else 4 for k in ("dtype", "y"))
        ids, ranks = _requests(c, 1)
        live, used = ids[ids >= 0], np.unique(ids[ids >= 0])
        return dict(bytes=4 * T + len(live) * c["Kd"] * esz + int(ranks[used].sum()) * (c["Kd"] + c["N"]) * esz + 8 * len(used) + 2 * T * c["N"] * ysz,
                    flops=2.0 * float(ranks[live].sum()) * (c["Kd"] + c["N"]))
    _, mask, table = _tables(c, 1)
    ids = _substitutes(mask, table)[_routed(c, 1)[0]].reshape(-1)
    rows, groups = int((ids >= 0).sum()), len(np.unique(ids[ids >= 0])) + c["shared"]
    d, F = c["d"], c["F"]
    matrix = d * F + 4 * -(-d // BLOCK) * -(-F // BLOCK) if c["experts"] == "q8" else 2 * d * F
    return dict(bytes=T * d * 4 + 8 * T * c["K"] + 4 * c["E"] * c["R"] + groups * 3 * matrix, flops=6.0 * (rows + c["shared"] * T) * d * F)


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    """8-bit values in the middle of a layer are rounded to e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6,
    halves to even; the operator's scale and the quotient in front of that rounding are 32-bit numbers by definition."""
    c = case
    s = prepare(case, seed)
    if c["kind"] == "route":
        z = s["x"].double() @ s["w_router"].double().T + s["bias"].double()
        p = torch.sigmoid(z) if c["scoring"] == "sigmoid" else torch.softmax(z, 1)
        v = p.clone() if s["balance"] is None else p + s["balance"].double()
        per = c["E"] // c["groups"]
        if c["keep"] < c["groups"]:
            best = torch.sort(v.view(c["T"], c["groups"], per), dim=2, descending=True).values[:, :, : c["top"]].sum(2)
            order = torch.argsort(best, dim=1, descending=True, stable=True)
            away = order[:, c["keep"]:]
            for g in range(away.shape[1]):
                v.scatter_(1, away[:, g: g + 1] * per + torch.arange(per, device=v.device), -math.inf)
        ids = torch.argsort(v, dim=1, descending=True, stable=True)[:, : c["K"]]
        live = torch.isfinite(v.gather(1, ids))
        w = p.gather(1, ids) * live
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return dict(ids=torch.where(live, ids, torch.full_like(ids, -1)).int(), w=w * c["scale"])
    if c["kind"] == "adapters":
        y = s["base"].double()
        ids, ranks = _requests(c, seed)
        for a in range(c["n"]):
            rows, r = torch.from_numpy(np.nonzero(ids == a)[0]).cuda(), int(ranks[a])
            if len(rows):
                y[rows] += float(s["scale"][a]) * ((s["x"][rows].double() @ s["a"][a, :r].double().T) @ s["b"][a, :, :r].double().T)
        return y
    T, K = c["T"], c["K"]
    q8 = c["experts"] == "q8"

    def spread(scale, width):
        return scale[..., torch.arange(width, device=scale.device) // BLOCK]

    def held(x):
        if not q8:
            return x
        most = torch.stack([x[..., k: k + BLOCK].abs().amax(-1) for k in range(0, x.shape[-1], BLOCK)], -1)
        scale = spread((most / torch.full_like(most, MOST)).clamp(min=TINY).float().double(), x.shape[-1])
        v = (x / scale).float().double()
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(v / step) * step * scale

    def matrix(qs, e):
        q = qs[0][e].double()
        return q * spread(qs[1][e].double(), q.shape[1])[torch.arange(q.shape[0], device=q.device) // BLOCK] if q8 else q

    def ffn(rows, gate, up, down):
        g = rows @ gate.T
        return held(g * torch.sigmoid(g) * (rows @ up.T)) @ down.T

    _, mask, table = _tables(c, seed)
    lut = [e if mask[e] else next((int(b) for b in table[e] if mask[b]), -1) for e in range(c["E"])]
    given, w = _routed(c, seed)
    ids, w = torch.tensor(lut, device="cuda")[torch.from_numpy(given).cuda().long()], torch.from_numpy(w).cuda().double()
    x = held(s["x"].double())
    y = torch.zeros((T, c["d"]), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        t, k = torch.nonzero(ids == e, as_tuple=True)
        if len(t):
            y.index_add_(0, t, ffn(x[t], matrix(s["gate"], e), matrix(s["up"], e), matrix(s["down"], e)) * w[t, k][:, None])
    for e in range(c["shared"]):
        y += ffn(x, *(matrix(m, e) for m in s["shared"]))
    return y
