"""Groups of which one expert or none can be taken: a group with none is behind every other."""
import numpy as np
import pytest
import torch

from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def taken(l, top_k, n_groups, kept):
    """ids of one token's scores by the definition: experts that can be taken, groups by (has such an expert, fp32 sum of the two best, lowest)."""
    groups = l.reshape(n_groups, -1)
    best = -np.sort(-groups, 1)[:, :2]
    score = best.sum(1, dtype=np.float32) if best.shape[1] == 2 else best[:, 0]
    order = sorted(range(n_groups), key=lambda g: (np.isneginf(best[g, 0]), -score[g], g))[:kept]
    ids = [e for e in np.argsort(-l, kind="stable") if not np.isneginf(l[e]) and e // groups.shape[1] in order][:top_k]
    return [int(e) for e in ids] + [-1] * (top_k - len(ids))


@pytest.mark.parametrize("E,G,kept,K", [(8, 4, 1, 2), (64, 8, 4, 8), (6, 6, 2, 3), (256, 64, 3, 8), (1024, 2, 1, 4)])
def test_groups_with_one_expert_left(E, G, kept, K):
    """From every expert but one masked to a few left, in every place of a group."""
    g, T = np.random.default_rng(E + G), 200
    l = g.standard_normal((T, E)).astype(np.float32)
    for t in range(T):
        some = g.choice(E, size=min(E, t % 7), replace=False)
        l[t, np.setdiff1d(np.arange(E), some)] = -np.inf
    l[7::14] = np.where(np.isneginf(l[7::14]), np.nan, l[7::14])
    want = np.array([taken(np.where(np.isnan(row), -np.inf, row).astype(np.float32), K, G, kept) for row in l])
    ctx = B.Context(1, E, K, 0, 8, B.MW_ROW_BF16, T, 0, np.zeros(E, dtype=np.int32))
    ids, w = torch.empty((T, K), dtype=torch.int32, device=DEV), torch.empty((T, K), device=DEV)
    for bias in (None, torch.zeros(E, device=DEV)):
        ctx.mw_route(B.Gate(B.MW_GATE_SOFTMAX_TOPK, G, kept), torch.from_numpy(l).to(DEV), bias, ids, w)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(ids.cpu().numpy(), want)
        alive = ~(np.isneginf(l) | np.isnan(l)).all(1)
        np.testing.assert_array_equal(ids.cpu().numpy()[:, 0] >= 0, alive)        # only a token whose experts are all masked goes nowhere
        assert np.abs(w.cpu().numpy().sum(1) - alive).max() <= 64 * 2.0 ** -24
    ctx.close()


def test_lowest_values_are_no_mask_of_a_group():
    """Two experts of the type's lowest value sum to -inf in fp32: their group is still ahead of one that is masked, and among such groups the
    lowest is taken."""
    low, E, G, K = float(torch.finfo(torch.float32).min), 16, 4, 3
    l = torch.full((3, E), -float("inf"), device=DEV)
    l[0, 8:12] = low
    l[1, 4:], l[1, 14] = low, -float("inf")
    l[2, 12:14], l[2, 5] = low, 1.0
    ctx = B.Context(1, E, K, 0, 8, B.MW_ROW_BF16, 3, 0, np.zeros(E, dtype=np.int32))
    ids, w = torch.empty((3, K), dtype=torch.int32, device=DEV), torch.empty((3, K), device=DEV)
    ctx.mw_route(B.Gate(B.MW_GATE_SOFTMAX_TOPK, G, 1), l, None, ids, w)
    torch.cuda.synchronize()
    assert ids.cpu().tolist() == [[8, 9, 10], [4, 5, 6], [5, -1, -1]]
    ctx.close()
