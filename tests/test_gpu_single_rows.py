"""A single row has no distance to a next one: views of one row are taken whatever their stride."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def one_row(t, stride):
    """[1, width] with `stride` elements to a next row that is not there."""
    return torch.as_strided(t, (1, t.shape[1]), (stride, 1))


@pytest.mark.parametrize("stride", [1, 67, 1 << 31])
def test_one_row(stride):
    g = torch.Generator().manual_seed(2)
    H, I, n, r = 64, 32, 4, 8
    x, dy = (torch.randn((1, H), generator=g).bfloat16() for _ in range(2))
    up, down, a, b = ((torch.randn(s, generator=g) * s[-1] ** -0.5).bfloat16() for s in ((n, 2, I, H), (n, H, I), (3, r, H), (3, H, r)))
    ctx = B.Context(1, n, 2, 0, H, B.MW_ROW_BF16, 1, 0, np.zeros(n, dtype=np.int32))
    experts, gate = B.Experts(up.to(DEV), down.to(DEV)), B.Gate(B.MW_GATE_SOFTMAX_TOPK)
    l = torch.randn((1, n), generator=g)
    ids, w, out = torch.empty((1, 2), dtype=torch.int32, device=DEV), torch.empty((1, 2), device=DEV), torch.empty((1, H), dtype=torch.bfloat16, device=DEV)
    ctx.mw_moe_layer(gate, one_row(l.to(DEV), stride), None, experts, one_row(x.to(DEV), stride), ids, w, one_row(out, stride), ctx.moe_workspace(experts, 1))
    want_ids, want_w = P.route(l.numpy(), None, 2, P.SOFTMAX_TOPK)
    assert (ids.cpu().numpy() == want_ids).all() and (np.abs(w.cpu().numpy() - want_w) <= 64 * 2.0 ** -24 * want_w).all()
    want, off = P.layer(x.double().numpy(), want_ids, w.cpu().numpy(), up.double().numpy(), down.double().numpy(), {i: i for i in range(n)}, 128 * 2.0 ** -24)
    assert (np.abs(out.float().cpu().numpy() - want) <= off + 2.0 ** -8 * np.abs(want)).all()

    gamma = 300 * 2.0 ** -24
    adapters, which = B.Adapters(a.to(DEV), b.to(DEV)), torch.tensor([1], dtype=torch.int32, device=DEV)
    ws, h, y, dx = adapters.workspace(1), torch.empty((1, r), device=DEV), torch.empty_like(out), torch.empty_like(out)
    adapters.mw_adapt(one_row(x.to(DEV), stride), which, one_row(dy.to(DEV), stride), one_row(y, stride), ws, h)
    da, db = torch.empty((3, r, H), dtype=torch.bfloat16, device=DEV), torch.empty((3, H, r), dtype=torch.bfloat16, device=DEV)
    adapters.mw_adapt_backward(one_row(x.to(DEV), stride), which, h, one_row(dy.to(DEV), stride), None, one_row(dx, stride), da, db, ws)
    plain = [t.double().numpy() for t in (x, dy, a, b)]
    want, _, off, _ = P.adapt(plain[0], [1], plain[1], plain[2], plain[3], np.ones(3), gamma)
    assert (np.abs(y.float().cpu().numpy() - want) <= off + 2.0 ** -8 * np.abs(want)).all()
    want = P.adapt_backward(plain[0], np.array([1]), h.double().cpu().numpy(), plain[1], np.zeros((1, H)), plain[2], plain[3], np.ones(3), gamma)
    for got, (v, off) in zip((dx, da, db), want):
        assert (np.abs(got.float().cpu().numpy() - v) <= off + 2.0 ** -8 * np.abs(v)).all()
    ctx.close()
