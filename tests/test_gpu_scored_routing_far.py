"""Routing by scores with logits far from zero, where an exponential's argument has no bits left for its fraction (needs an MI355X)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

T, E = 64, 32


def route(z, scoring):
    """All experts' ids and scores: tokens are unit vectors and the router holds the logits, which are exact then."""
    import torch
    import paper_2511_10054_amd as bm
    desc = bm.RouterDesc(T=T, d=T, E=E, K=E, n_groups=1, keep_groups=1, group_top=1, scoring=getattr(bm, "BM_SCORE_" + scoring.upper()),
                         dtype=bm.BM_F32, flags=0, scale=1.0)
    x, w = torch.eye(T, device="cuda"), torch.from_numpy(np.ascontiguousarray(z.T.astype(np.float32))).cuda()
    ids, weights = torch.empty((T, E), dtype=torch.int32, device="cuda"), torch.empty((T, E), device="cuda")
    bm.bm_route_scored(desc, x, w, None, None, ids, weights, torch.empty(bm.bm_workspace_bytes_scored(desc), dtype=torch.uint8, device="cuda"))
    return ids.cpu().numpy(), weights.double().cpu().numpy()


# An exponential: the instruction's unit in the last place (2 * 2^-24), the product with what its argument has no room for, rounded once (1);
# one more addition (1); a reciprocal's unit in the last place (2), or a division and a product (2).  All above 2^-126.  Second order: 1.
TOL = 7 * 2.0 ** -24


@pytest.mark.parametrize("scoring", ["sigmoid", "softmax"])
@pytest.mark.parametrize("lo,hi", [(-87.1875, -83.0), (-83.0, -40.0), (-87.1875, 8.0)])
def test_scores_down_to_the_smallest_normal_number(scoring, lo, hi):
    """To the precision of the numbers; 87.1875 = 126 log 2 - 0.15."""
    g = np.random.default_rng(11)
    grid = np.arange(lo, hi, 2.0 ** -6)                                        # apart by 2^-6: no rounding turns the order
    z = np.stack([g.choice(grid, E, replace=False) for _ in range(T)])
    if scoring == "softmax":
        z[:, 5] = 0.0                                                          # the largest (or one of the largest)
        z[:, :5] = np.minimum(z[:, :5], 0.0) + np.where(z[:, :5] >= 0, lo / 2 + np.arange(5) / 8, 0.0)
        z = np.minimum(z, 0.0)
        for t in range(T):                                                     # one zero a token
            again = np.nonzero(z[t] == 0)[0]
            z[t, again] = np.where(again == 5, 0.0, lo / 3 - 2.0 ** -7 * (1 + np.arange(len(again))))
        s = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    else:
        s = 1.0 / (1.0 + np.exp(-z))
    ids, w = route(z, scoring)
    want = np.argsort(-z, axis=1, kind="stable")
    np.testing.assert_array_equal(ids, want)
    # (a sum of 32 softmax terms below the largest: their own errors, and 12 more roundings of what they add to 1)
    np.testing.assert_allclose(w, np.take_along_axis(s, want, 1), rtol=TOL + (12 * 2.0 ** -24 if scoring == "softmax" else 0), atol=0)


def test_sigmoids_that_are_equal_in_32_bits_go_by_index():
    """1 / (1 + e^-z) rounds to 1 where e^-z is under half a step below 1, 2^-25: for z above 25 log 2 = 17.33."""
    z = np.tile(np.linspace(-3.0, 3.0, E), (T, 1))
    z[:, [4, 9, 20, 30]] = [18.0, 40.0, 25.0, 87.0]
    ids, w = route(z, "sigmoid")
    assert (ids[:, :4] == [4, 9, 20, 30]).all() and (w[:, :4] == 1).all()
    rest = [e for e in range(E - 1, -1, -1) if e not in (4, 9, 20, 30)]
    assert (ids[:, 4:] == rest).all()


@pytest.mark.parametrize("scoring", [0, 1])
@pytest.mark.parametrize("E,G", [(40, 4), (32, 4), (128, 4), (256, 8), (255, 5)])
def test_a_groups_score_that_is_no_number(E, G, scoring):
    """The sum of an infinite choice and one of -infinity counts as -infinity: the group comes behind every group with a number, and after a
    lower group of -infinity."""
    import torch
    import paper_2511_10054_amd as bm
    per, K, INF = E // G, 4, float("inf")
    gen = torch.Generator(device="cuda").manual_seed(E)
    x, w = torch.randn((3, 32), generator=gen, device="cuda").bfloat16(), torch.randn((E, 32), generator=gen, device="cuda").bfloat16()
    desc = bm.RouterDesc(T=3, d=32, E=E, K=K, n_groups=G, keep_groups=1, group_top=2, scoring=scoring, dtype=bm.BM_BF16, flags=bm.BM_RENORM_TOPK, scale=1.0)
    work = torch.empty(bm.bm_workspace_bytes_scored(desc), dtype=torch.uint8, device="cuda")

    def call(balance):
        ids, weights = torch.full((3, K), -9, dtype=torch.int32, device="cuda"), torch.full((3, K), -9.0, device="cuda")
        bm.bm_route_scored(desc, x, w, None, balance, ids, weights, work)
        return ids.cpu().numpy(), weights.cpu().numpy()

    b = torch.full((E,), -INF, device="cuda")
    b[per + 3] = INF                                           # of group 1; group 2 has finite choices
    b[2 * per: 3 * per] = -5.0
    ids, weights = call(b)
    assert ((ids >= 2 * per) & (ids < 3 * per)).all() and abs(weights.sum(1) - 1).max() < 1e-6
    b[2 * per: 3 * per] = -INF                                  # nothing else: group 0 is as good, and lower
    ids, weights = call(b)
    assert (ids == -1).all() and (weights == 0).all()
    b[per + 4] = -1.0                                           # with a number beside it the infinity counts
    b[2 * per: 3 * per] = 100.0
    ids, weights = call(b)
    assert (ids[:, :2] == [per + 3, per + 4]).all() and (ids[:, 2:] == -1).all()
