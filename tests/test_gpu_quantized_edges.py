"""Calls of the 8-bit operators that the documentation allows at its edges: groups that begin behind row 0, scales and maps at any
4-byte address, the most groups there are, shared experts alone (needs an MI355X)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, product_error
from test_gpu_quantized import check_swiglu
from test_gpu_quantized_layer import LIMIT, Quantized
from test_gpu_quantized_tiles import FORTY, SIXTY, Operands, mixed

pytestmark = pytest.mark.gpu


def at_odd_address(t):
    """The same values 4 bytes past a 16-byte boundary, poison around them."""
    room = torch.full((t.numel() + 8,), float("nan") if t.is_floating_point() else -(1 << 30), dtype=t.dtype, device=t.device)
    view = room[1:1 + t.numel()].view(t.shape)
    view.copy_(t)
    assert view.data_ptr() % 16 == 4
    return view


# single products of few rows, tiles of 32 (whole reductions, in parts), 64, 128 and 192 rows
SHAPES = [([5, 0, 2], 160, 2048, 2), (mixed(64, 12, 5), 1056, 512, 3), (mixed(16, 12, 1), 800, 2176, 2), (FORTY, 2816, 2176, 1), (SIXTY, 3200, 352, 2),
          ([600, 0, 700], 8224, 480, 2), ([300, 250, 280], 4128, 512, 3)]


@pytest.mark.parametrize("counts,N,Kd,K", SHAPES)
def test_groups_behind_row_zero(counts, N, Kd, K):
    """The first group begins at row 37: rows before it are left as they were, and so are those behind the last."""
    print("behind row zero", sum(counts), len(counts), N, Kd, K, flush=True)
    first, slack = 37, 6
    rows = sum(counts)
    o = Operands(counts, N, Kd, -(-rows // K) + first + slack, matrices=2, K=K)
    offsets = at_odd_address(o.offsets + first)
    ids = o.map if o.map is not None else o.src.int()
    ids = at_odd_address(torch.cat([torch.full((first,), -1, dtype=torch.int32, device="cuda"), ids, torch.full((slack,), -1, dtype=torch.int32, device="cuda")]))
    sa, (gate, gs), (up, us) = at_odd_address(o.sa), *((q, at_odd_address(s)) for q, s in o.w)
    live = slice(first, first + rows)
    for dtype, code in ((torch.float32, bm.BM_F32), (torch.bfloat16, bm.BM_BF16)):
        c = torch.full((first + rows + slack, N), -7.0, dtype=dtype, device="cuda")
        bm.bm_grouped_matmul(o.desc(first + rows + slack, code), o.a, sa, ids, offsets, gate, gs, c)
        want, absolute = o.exact()
        bound = product_error(absolute, Kd)
        if dtype == torch.bfloat16:
            # eight products at once, each cut below 2^-13 of the largest; bf16's half step
            bound = bound + 2.0 ** -8 * want.abs() + 2.0 ** -10 * 1.01 * absolute
        assert bool(((c[live].double() - want).abs() <= bound + 1e-30).all())
        assert bool((c[:first] == -7.0).all()) and bool((c[first + rows:] == -7.0).all())
    h, s = torch.full((first + rows + slack, N), 0x55, dtype=torch.uint8, device="cuda"), at_odd_address(torch.full((first + rows + slack, -(-N // BLOCK)), -7.0, device="cuda"))
    bm.bm_grouped_swiglu(o.desc(first + rows + slack), o.a, sa, ids, offsets, gate, gs, up, us, h, s)
    (wg, ag), (wu, au) = o.exact(0), o.exact(1)
    check_swiglu(h[live].cpu().numpy(), s[live].cpu().numpy(), *(t.cpu().numpy() for t in (wg, wu, product_error(ag, Kd), product_error(au, Kd))), N)
    for part in (slice(0, first), slice(first + rows, None)):
        assert bool((h[part] == 0x55).all()) and bool((s[part] == -7.0).all())


def test_layer_with_the_most_groups():
    """256 experts and 8 shared ones: as many groups as a table of tiles holds."""
    print("264 groups", flush=True)
    L = Quantized("c4_qwen3", dict(d=96, E=256, F=64, n_resident=200, n_shared=8), 70)
    out = {k: v.cpu().numpy() for k, v in L.forward().items()}
    ref = L.host.oracle_forward(oracle)
    np.testing.assert_array_equal(out["ids_remapped"], ref["ids_remapped"])
    want = L.reference(ref["ids_remapped"], ref["w"].astype(np.float64))
    assert np.linalg.norm(L.y.double().cpu().numpy() - want) <= LIMIT * np.linalg.norm(want)


@pytest.mark.parametrize("T", [5, 300])
def test_shared_experts_alone(T):
    """No routed expert is resident: y is the shared experts' sum, and no routed weight is read."""
    print("shared alone", T, flush=True)
    L = Quantized("c5_deepseek", dict(d=256, F=160), T)
    for t in L.dev[:6]:
        t.fill_(0x7f if t.dtype == torch.uint8 else float("nan"))
    L.bitmap.zero_()
    dbg = L.forward()
    assert (dbg["ids_remapped"] == -1).all() and (dbg["offsets"] == 0).all()
    want = L.reference(np.full((T, L.spec.K), -1), np.zeros((T, L.spec.K)))
    assert np.linalg.norm(L.y.double().cpu().numpy() - want) <= LIMIT * np.linalg.norm(want)


def test_two_graphs_with_workspaces_of_their_own():
    """Two captured layers replayed at once on two streams, and again on new tokens."""
    print("two graphs", flush=True)
    layers = [Quantized("c4_qwen3", dict(d=512, E=32, F=1408, K=4, n_resident=32), 64), Quantized("c5_deepseek", dict(d=256, F=352), 300)]
    graphs = []
    for L in layers:
        L.forward(debug=False)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            L.forward(debug=False)
    streams = [torch.cuda.Stream() for _ in layers]
    for turn in range(3):
        for L in layers:
            L.x.copy_(L.x.flip(0).clone())
            L.y.zero_()
            L.work.fill_(0xA5)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        replayed = [L.y.clone() for L in layers]
        for L, y in zip(layers, replayed):
            L.y.zero_()
            L.forward(debug=False)
            assert torch.equal(L.y, y) and bool(torch.isfinite(y.float()).all()), turn
