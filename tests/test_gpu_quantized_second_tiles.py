"""Gathered gate/up products whose workgroups take a second tile on four stages, from the shortest reductions on: rows, ids and
scales of the next tile are fetched under the present one (needs an MI355X)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2511_10054_amd as bm
from helpers_8bit import BLOCK, product_error
from test_gpu_quantized import check_swiglu
from test_gpu_quantized_layer import LIMIT, Quantized
from test_gpu_quantized_tiles import Operands, a_rows_of

pytestmark = pytest.mark.gpu

SMALL = [8] * 64
UNEVEN = [0, 1, 33, 17, 16, 2, 0, 31] * 8          # live groups of 1 to 33 rows: one tile, and two
CASES = [
    (SMALL, 640, 512, 4), (SMALL, 640, 480, 4), (SMALL, 640, 416, 8), (SMALL, 640, 96, 2), (SMALL, 640, 32, 3),      # walks of four steps
    ([8] * 32, 1408, 512, 4), (UNEVEN, 640, 512, 6), (UNEVEN, 608, 352, 2),
    (SMALL, 640, 640, 4), (SMALL, 640, 608, 4), (UNEVEN, 640, 768, 4), (SMALL, 640, 1024, 4),                        # of five, six and eight
    (SMALL, 1408, 4096, 4), (SMALL, 1408, 4128, 2),                                                                 # up to four tiles a unit
]


def tiles(counts, N):
    """(32-row tiles that there are, the most of any grouping of these rows)"""
    return sum(-(-n // 32) for n in counts) * -(-N // BLOCK), (sum(counts) // 32 + len(counts)) * -(-N // BLOCK)


def check_case(o, h, s):
    (wg, ag), (wu, au) = o.exact(0), o.exact(1)
    wg, ag, wu, au = (t.cpu().numpy() for t in (wg, ag, wu, au))
    check_swiglu(h[:o.rows].cpu().numpy(), s[:o.rows].cpu().numpy(), wg, wu, product_error(ag, o.Kd), product_error(au, o.Kd), o.N)


@pytest.mark.parametrize("counts,N,Kd,K", CASES)
def test_second_tiles_read_their_own_rows(counts, N, Kd, K):
    print("second tiles", sum(counts), len(counts), N, Kd, K, flush=True)
    real, bound = tiles(counts, N)
    assert real > 256 and bound <= (1024 if Kd >= 4096 else 512) and sum(counts) // len(counts) < 32        # four stages, a unit each
    o = Operands(counts, N, Kd, a_rows_of(counts, K), matrices=2, K=K)
    h, s = o.swiglu(slack=4)
    assert bool((h[o.rows:] == 0x55).all()) and bool((s[o.rows:] == -7.0).all())
    check_case(o, h, s)
    other = Operands(SMALL, 640, 512, a_rows_of(SMALL, 4), matrices=2, K=4, seed=9)                         # leaves its ids in LDS
    for _ in range(3):
        other.swiglu()
        again = o.swiglu(slack=4)
        assert torch.equal(again[0], h) and torch.equal(again[1], s)


def test_gathered_calls_on_two_streams_at_once():
    print("two streams, gathered", flush=True)
    sets = [Operands(c, N, Kd, a_rows_of(c, K), matrices=2, K=K, seed=i) for i, (c, N, Kd, K) in enumerate(CASES[:8:2] + CASES[8:11])]
    alone = [(o.product(torch.float32), o.product(torch.bfloat16), *o.swiglu()) for o in sets]
    for o, (_, _, h, s) in zip(sets, alone):
        check_case(o, h, s)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for k, st in enumerate(streams):
        with torch.cuda.stream(st):
            for o in (sets if k == 0 else sets[::-1]):
                got[k].append((o.product(torch.float32), o.product(torch.bfloat16), *o.swiglu()))
    torch.cuda.synchronize()
    for results in (got[0], got[1][::-1]):
        for one, two in zip(alone, results):
            assert all(torch.equal(x, y) for x, y in zip(one, two))


@pytest.mark.parametrize("T,d", [(64, 512), (64, 96), (50, 480), (60, 640)])
def test_layer_of_many_small_experts(T, d):
    """32 resident experts of 1408 columns, four a token, hidden sizes from the shortest on: more than 256 tiles of gate and up."""
    print("many small experts", T, d, flush=True)
    L = Quantized("c4_qwen3", dict(d=d, E=32, F=1408, K=4, n_resident=32), T)
    out = {k: v.cpu().numpy() for k, v in L.forward().items()}
    real, bound = tiles(np.diff(out["offsets"]).tolist(), 1408)
    assert real > 256 and bound <= 512
    ref = L.host.oracle_forward(oracle)
    np.testing.assert_array_equal(out["ids_remapped"], ref["ids_remapped"])
    want = L.reference(ref["ids_remapped"], ref["w"].astype(np.float64))
    rel = np.linalg.norm(L.y.double().cpu().numpy() - want) / np.linalg.norm(want)
    print("   rel", rel, flush=True)
    assert rel <= LIMIT
    y = L.y.clone()
    L.work.fill_(0xFF)
    L.forward(debug=False)
    assert torch.equal(L.y, y)
