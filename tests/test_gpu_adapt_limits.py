"""Calls at the limits of the adapters and the experts."""
import numpy as np
import pytest
import torch

from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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
