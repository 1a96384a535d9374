"""Calls of the experts that are within the stated limits and are taken."""
import ctypes as C

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


@pytest.mark.parametrize("hidden,inter,fp8,status", [(32768, 32768, True, B.MW_OK), (32768, 24576, True, B.MW_OK), (32768, 32784, True, B.MW_ERR_UNSUPPORTED),
                                                     (32768, 16384, False, B.MW_OK), (32768, 16392, False, B.MW_ERR_UNSUPPORTED)])
def test_an_experts_gate_and_up_span_2_gib(hidden, inter, fp8, status):
    """Calls without tokens, which check their arguments and launch nothing."""
    ctx = B.Context(1, 2, 1, 0, hidden, B.MW_ROW_BF16, 4, 0, np.zeros(2, dtype=np.int32))
    some, ws, need = torch.zeros(256, device=DEV), torch.zeros(4096, dtype=torch.uint8, device=DEV), C.c_int64(0)
    at = some.data_ptr()
    rec = B.MwExperts(at, at, at if fp8 else 0, at if fp8 else 0, inter, B.MW_ROW_FP8_E4M3_BLOCK128 if fp8 else B.MW_ROW_BF16)
    assert B.load().mw_moe_workspace_bytes(ctx._h, C.byref(rec), C.c_int32(4), C.byref(need)) == B.MW_OK
    ws = ws[(-ws.data_ptr()) % 256:]
    assert B._native().mw_moe_layer(ctx._h, 0, None, 0, 0, None, C.addressof(rec), some, hidden, 0, some, some, some, hidden, None, ws, ws.numel(), 0) == status
    ctx.close()


def test_an_expert_of_2_gib():
    """Two tokens through an fp8 expert whose gate and up rows end 2 GiB from their start; 64-bit products a piece of rows at a time.  A wave adds up 64
    spans of four instructions and a factor: 300 u of the sum of sizes, u = 2^-24, covers it; the activation's split 2^-15, the output's rounding 2^-8."""
    H = I = 32768
    u, g = 300 * 2.0 ** -24, torch.Generator(device=DEV).manual_seed(1)
    ctx = B.Context(1, 1, 1, 0, H, B.MW_ROW_BF16, 2, 0, np.zeros(1, dtype=np.int32))
    codes = [torch.randint(0, 255, s, generator=g, device=DEV, dtype=torch.uint8) for s in ((1, 2, I, H), (1, H, I))]
    for c in codes:
        c[(c & 0x7f) == 0x7f] = 0                                       # (no NaN)
        c.bitwise_and_(0xb7)                                            # (values up to 1.875)
    up, down = (c.view(torch.float8_e4m3fn) for c in codes)
    scales = [torch.rand(s, generator=g, device=DEV) * 0.02 + 0.005 for s in ((1, 2, I // 128, H // 128), (1, H // 128, I // 128))]
    x = torch.randn((2, H), generator=g, device=DEV).bfloat16()

    def product(codes, scale, v, off):
        """(codes v, the size of its error where v is off by `off`); v, off [columns][2]"""
        out, err = [], []
        for r in range(0, codes.shape[0], 2048):
            w = codes[r:r + 2048].double() * scale[r // 128:(r + 2048) // 128].double().repeat_interleave(128, 0).repeat_interleave(128, 1)
            out.append(w @ v)
            err.append(w.abs() @ (u * v.abs() + off))
        return torch.cat(out), torch.cat(err)

    xs = x.double().t().contiguous()
    (a, da), (b, db) = (product(up[0, i], scales[0][0, i], xs, xs * 0) for i in range(2))
    act = a / (1 + torch.exp(-a)) * b
    d_act = 1.1 * b.abs() * da + (a / (1 + torch.exp(-a))).abs() * db + 1.1 * da * db + 2.0 ** -15 * act.abs()
    want, off = product(down[0], scales[1][0], act, d_act)
    out = torch.empty((2, H), dtype=torch.bfloat16, device=DEV)
    experts = B.Experts(up, down, *scales)
    ids, w = torch.zeros((2, 1), dtype=torch.int32, device=DEV), torch.ones((2, 1), device=DEV)
    ctx.mw_moe_layer(None, None, None, experts, x, ids, w, out, ctx.moe_workspace(experts, 2))
    torch.cuda.synchronize()
    assert ((out.double().t() - want).abs() <= off + 2.0 ** -8 * want.abs()).all()
    assert off.max() < 0.5 * want.square().mean().sqrt()                # (weights from elsewhere would be off by more)
    ctx.close()
