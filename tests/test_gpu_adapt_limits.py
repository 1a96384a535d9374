"""Calls at the adapters' limits: factors of more pieces than one dimension of a grid has, strides whose product with the rows passes 64 bits."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B
from test_gpu_adapt import DEV, GAMMA, close, normal

pytestmark = pytest.mark.gpu


def test_gradients_of_very_wide_projections():
    """1024 adapters of rank 8 to 262144 values: more than 2^32 threads would transpose a piece of the factors each."""
    n, rank, n_in, n_out, used = 1024, 8, 8, 262144, [3, 700, 1023]
    a, b = torch.zeros((n, rank, n_in), dtype=torch.bfloat16, device=DEV), torch.zeros((n, n_out, rank), dtype=torch.bfloat16, device=DEV)
    some_a, some_b = normal(1, 3, rank, n_in).bfloat16(), (normal(2, 3, n_out, rank) * rank ** -0.5).bfloat16()
    a[used], b[used] = some_a.to(DEV), some_b.to(DEV)
    ids, order = torch.tensor([1023, 3, 700, 3], dtype=torch.int32), np.array([2, 0, 1, 0])
    x, dy, h = normal(5, 4, n_in).bfloat16(), normal(6, 4, n_out).bfloat16(), normal(8, 4, rank)
    adapters = B.Adapters(a, b)
    dx, da, db = torch.empty((4, n_in), dtype=torch.bfloat16, device=DEV), torch.full_like(a, 7.0), torch.full_like(b, 7.0)
    adapters.mw_adapt_backward(x.to(DEV), ids.to(DEV), h.to(DEV), dy.to(DEV), None, dx, da, db, adapters.workspace(4))
    torch.cuda.synchronize()
    # sums over 262144 values in eight slices of four waves: 8192 values a wave, an instruction adds 32 of them
    want = P.adapt_backward(x.double().numpy(), order, h.double().numpy(), dy.double().numpy(), np.zeros((4, n_in)), some_a.double().numpy(),
                            some_b.double().numpy(), np.ones(3), GAMMA)
    for got, (v, off) in zip((dx, da[used], db[used]), want):
        close(got.float().cpu().numpy(), v, off)
    da[used], db[used] = 0, 0
    assert not da.any() and not db.any()


def test_strides_that_pass_64_bits_with_the_rows():
    H, n, T = 64, 2, 8
    x, out, h = torch.zeros((T, H), dtype=torch.bfloat16, device=DEV), torch.zeros((T, H), dtype=torch.bfloat16, device=DEV), torch.zeros((T, 16), device=DEV)
    ids, a, b = torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros((n, 16, H), dtype=torch.bfloat16, device=DEV), torch.zeros((n, H, 16), dtype=torch.bfloat16, device=DEV)
    adapters, da, db = B.Adapters(a, b), torch.empty_like(a), torch.empty_like(b)
    ws, far = adapters.workspace(T), 1 << 61
    fwd = [adapters.address, x, H, ids, T, out, H, out, H, None, None, ws, ws.numel(), 0]
    back = [adapters.address, x, H, ids, T, h, out, H, x, H, x, H, da, db, None, ws, ws.numel(), 0]
    for call, good, places in ((B._native().mw_adapt, fwd, (2, 6, 8)), (B._native().mw_adapt_backward, back, (2, 7, 9, 11))):
        assert call(*good) == B.MW_OK
        for at in places:
            for stride in (far, 1 << 62, (1 << 27) + 8):
                assert call(*(good[:at] + [stride] + good[at + 1:])) == B.MW_ERR_UNSUPPORTED, (at, stride)
    ctx = B.Context(1, n, 1, 0, H, B.MW_ROW_BF16, T, 0, np.zeros(n, dtype=np.int32))
    experts = B.Experts(torch.zeros((n, 2, 16, H), dtype=torch.bfloat16, device=DEV), torch.zeros((n, H, 16), dtype=torch.bfloat16, device=DEV))
    ws, w = ctx.moe_workspace(experts, T), torch.zeros((T, 1), device=DEV)
    good = [ctx._h, 0, None, 0, 0, None, experts.address, x, H, T, ids, w, out, H, None, ws, ws.numel(), 0]
    assert B._native().mw_moe_layer(*good) == B.MW_OK
    for stride in (far, 1 << 62, (1 << 27) + 8):
        assert B._native().mw_moe_layer(*(good[:8] + [stride] + good[9:])) == B.MW_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    ctx.close()
