"""Calls of the experts that are within the stated limits and are taken."""
import numpy as np
import pytest
import torch

from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T", [0, 3, 40])
def test_a_rank_without_fp8_experts_writes_zeros(T):
    E, H, I = 8, 128, 64
    ctx = B.Context(4, E, 2, 3, H, B.MW_ROW_BF16, 64, 0, np.zeros(E, dtype=np.int32))
    none = [torch.empty((0,) + s, dtype=d, device=DEV) for s, d in (((2, I, H), torch.float8_e4m3fn), ((H, I), torch.float8_e4m3fn), ((2, 1, 1), torch.float32), ((1, 1), torch.float32))]
    experts = B.Experts(*none)
    out = torch.full((T + 1, H), 7.0, dtype=torch.bfloat16, device=DEV)
    ids, w = torch.randint(0, E, (T, 2), device=DEV).int(), torch.ones((T, 2), device=DEV)
    ctx.mw_moe_layer(None, None, None, experts, torch.ones((T, H), dtype=torch.bfloat16, device=DEV), ids, w, out[:T], ctx.moe_workspace(experts, T))
    torch.cuda.synchronize()
    assert (out[:T] == 0).all() and (out[T] == 7).all()
    ctx.close()
