"""Sigmoid gates whose chosen scores are all far below zero: sig(l) itself is below fp32's range there, the shares are not.

Tolerances, u = 2^-24, as in the gate's other tests: a share is exp of a difference of at most 30 (off by 30 u), the function, a quotient and a
sum: 64 u.  The gradient adds one more such share and a difference: 128 u of the sizes of what is added up."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, TINY = 2.0 ** -24, 2.0 ** -126
E, K, SCALE = 48, 6, 2.5
LEVELS = (0.0, -60.0, -80.0, -88.0, -90.0, -104.0, -200.0, -680.0)


def rows():
    """A row a level, scores within 20 of it; one with a score far above the rest, one of whose experts only the low ones are left."""
    g = torch.Generator().manual_seed(3)
    l = torch.stack([level + 20.0 * torch.rand(E, generator=g) - 10.0 for level in LEVELS + (-120.0, -120.0)])
    l[-2, 7] = 3.0
    l[-1, 3:] = -float("inf")
    return l


def route(l, dw=None, gate=None):
    ctx = B.Context(1, l.shape[1], K, 0, 8, B.MW_ROW_BF16, len(l), 0, np.zeros(l.shape[1], dtype=np.int32))
    gate, l = gate or B.Gate(B.MW_GATE_SIGMOID_TOPK, scale=SCALE), l.to(DEV)
    ids, w, d = torch.empty((len(l), K), dtype=torch.int32, device=DEV), torch.empty((len(l), K), device=DEV), torch.empty_like(l)
    ctx.mw_route(gate, l, None, ids, w)
    if dw is not None:
        ctx.mw_route_backward(gate, l, ids, dw.to(DEV), d)
    torch.cuda.synchronize()
    ctx.close()
    return ids.cpu().numpy(), w.cpu().numpy(), d.float().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shares_of_low_scores(dtype):
    l = rows().to(dtype)
    ids, w, _ = route(l)
    want_ids, want = P.route(l.float().numpy(), None, K, P.SIGMOID_TOPK, scale=SCALE)
    np.testing.assert_array_equal(ids, want_ids)
    assert (np.abs(want.sum(1) - SCALE) < 1e-9).all()                   # (no row of these is masked)
    assert (np.abs(w - want) <= 64 * U * np.abs(want) + TINY).all(), np.abs(w - want).max(1)


def test_gradient_of_low_scores():
    l, dw = rows(), torch.randn((len(LEVELS) + 2, K), generator=torch.Generator().manual_seed(4))
    ids, _, d = route(l, dw)
    want, size = P.route_backward(l.numpy(), ids, dw.numpy(), P.SIGMOID_TOPK, SCALE)
    assert (np.abs(want)[1:-2].max(1) > 1e-2).all()                     # (what is lost where the shares are)
    assert (np.abs(d - want) <= 128 * U * size + TINY).all(), np.abs(d - want).max(1)


@pytest.mark.parametrize("mask", [-1e4, -65504.0, float(torch.finfo(torch.bfloat16).min), float(torch.finfo(torch.float32).min)])
def test_values_that_stand_for_a_mask_weigh_nothing(mask):
    """Finite scores so low that sig(l) is no number of 64 bits either: chosen where nothing else is left, without a weight."""
    l = torch.full((3, E), mask)
    l[1, 5], l[2, :8] = -95.0, torch.arange(8) - 95.0
    dw = torch.randn((3, K), generator=torch.Generator().manual_seed(4))
    ids, w, d = route(l, dw)
    want_ids, want = P.route(l.numpy(), None, K, P.SIGMOID_TOPK, scale=SCALE)
    np.testing.assert_array_equal(ids, want_ids)
    assert (w[0] == 0).all() and (d[0] == 0).all() and w[1, 0] == SCALE and (w[1, 1:] == 0).all()
    assert (np.abs(w - want) <= 64 * U * np.abs(want) + TINY).all()
    want, size = P.route_backward(l.numpy(), ids, dw.numpy(), P.SIGMOID_TOPK, SCALE)
    assert (np.abs(d - want) <= 128 * U * size + TINY).all()


def test_a_token_with_low_scores_reaches_its_experts():
    """The layer's output is the experts' weighted sum, not zeros."""
    n, H, I = 4, 64, 32
    g = torch.Generator().manual_seed(6)
    up, down, x = ((torch.randn(s, generator=g) * s[-1] ** -0.5).bfloat16() for s in ((n, 2, I, H), (n, H, I), (2, H)))
    ctx = B.Context(1, n, 2, 0, H, B.MW_ROW_BF16, 2, 0, np.zeros(n, dtype=np.int32))
    experts = B.Experts(up.to(DEV), down.to(DEV))
    l = torch.tensor([[-91.0, -89.0, -90.0, -300.0], [1.0, -2.0, 0.5, 0.0]], device=DEV)
    ids, w, out = torch.empty((2, 2), dtype=torch.int32, device=DEV), torch.empty((2, 2), device=DEV), torch.empty((2, H), dtype=torch.bfloat16, device=DEV)
    ctx.mw_moe_layer(B.Gate(B.MW_GATE_SIGMOID_TOPK), l, None, experts, x.to(DEV), ids, w, out, ctx.moe_workspace(experts, 2))
    torch.cuda.synchronize()
    want_ids, want_w = P.route(l.cpu().numpy(), None, 2, P.SIGMOID_TOPK)
    assert (np.abs(w.cpu().numpy() - want_w) <= 64 * U * want_w).all()
    want, off = P.layer(x.double().numpy(), want_ids, w.cpu().numpy(), up.double().numpy(), down.double().numpy(), {i: i for i in range(n)}, 128 * U)
    assert (np.abs(want).max(1) > 0.01).all() and (np.abs(out.float().cpu().numpy() - want) <= off + 2.0 ** -8 * np.abs(want)).all()
    ctx.close()
