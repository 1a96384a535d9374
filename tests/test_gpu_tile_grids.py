"""Launches of more workgroups than fit one axis of a grid: tiles and gradients of many matrices."""
import itertools

import numpy as np
import pytest
import torch

import plain_experts as P
from paper_2605_22428_amd import binding as B
from test_gpu_ffn import DEV, host, near, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _leave_no_cache():
    yield
    torch.cuda.empty_cache()


def _room(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip("%.0f GiB of device memory free, %d needed" % (free / 2 ** 30, gib))


def test_tiles_that_lie_in_several_rows_of_the_grid():
    """17 rows in each of 2048 matrices 16 -> 69632: 1.1 million tiles of 128 x 64 with rows, 1.4 million workgroups.  Sums of 16 products of codes are exact, one rounding to bf16 is left."""
    _room(16)
    n, n_out, rows = 2048, 69632, 17
    w = torch.randint(-127, 128, (n, n_out, 16), dtype=torch.int8, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    codes = torch.randint(-127, 128, (n * rows, 16), dtype=torch.int8, device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    out = torch.full((n * rows, n_out), 7.0, dtype=torch.bfloat16, device=DEV)
    B.MatricesInt8(w, torch.ones((n, n_out), device=DEV)).mw_matmul_int8(codes, torch.ones(n * rows, device=DEV), torch.arange(n + 1, device=DEV) * rows, out)
    for m in range(0, n, 64):
        want = torch.matmul(codes[m * rows:(m + 64) * rows].float().view(64, rows, 16), w[m:m + 64].float().transpose(1, 2).contiguous())
        assert torch.equal(out[m * rows:(m + 64) * rows].view(64, rows, n_out), want.bfloat16()), m


def test_more_workgroups_than_a_launch_takes_along_an_axis():
    """26241 rows of room and 1640 matrices 16 -> 2^20 may be 2050 x 8192 tiles, above 2^24: three matrices have rows."""
    _room(110)
    n, n_out, room = 1640, 1 << 20, 16 * 1640 + 1
    counts = {0: 5, 819: 70, 1639: 1}
    w, scale = torch.empty((n, n_out, 16), dtype=torch.int8, device=DEV), torch.empty((n, n_out), device=DEV)
    g = torch.Generator(DEV).manual_seed(3)
    for m in counts:
        w[m] = torch.randint(-127, 128, (n_out, 16), dtype=torch.int8, device=DEV, generator=g)
        scale[m] = 1.0
    rows = sum(counts.values())
    codes = torch.randint(-127, 128, (room, 16), dtype=torch.int8, device=DEV, generator=g)
    out = torch.empty((room, n_out), dtype=torch.bfloat16, device=DEV)
    out[rows:rows + 64] = 7.0
    offsets = torch.tensor([0] + list(itertools.accumulate(counts.get(m, 0) for m in range(n))), device=DEV)
    B.MatricesInt8(w, scale).mw_matmul_int8(codes, torch.ones(room, device=DEV), offsets, out)
    first = 0
    for m, c in counts.items():
        assert torch.equal(out[first:first + c], (codes[first:first + c].float() @ w[m].float().T).bfloat16()), m
        first += c
    assert (out[rows:rows + 64] == 7).all()


def test_gradients_whose_tiles_lie_in_several_rows_of_the_grid():
    """65536 experts 1032 x 8: two million workgroups for their matrices' gradients, of which a few experts' have rows."""
    _room(24)
    n, hidden, inter = 65536, 1032, 8
    counts = {0: 3, 40000: 90, 65535: 2}
    rows = sum(counts.values())
    ctx = B.Context(1, n, 1, 0, hidden, B.MW_ROW_BF16, 1, rows, np.zeros(n, dtype=np.int32))
    gate_up, down = torch.zeros((n, 2, inter, hidden), dtype=torch.bfloat16, device=DEV), torch.zeros((n, hidden, inter), dtype=torch.bfloat16, device=DEV)
    for i, e in enumerate(counts):
        gate_up[e], down[e] = (normal(i, 2, inter, hidden) * hidden ** -0.5).bfloat16(), (normal(9 + i, hidden, inter) * inter ** -0.5).bfloat16()
    experts, offsets = B.Experts(gate_up, down), torch.tensor([0] + list(itertools.accumulate(counts.get(e, 0) for e in range(n))), device=DEV)
    x, dy, kept = normal(20, rows, hidden).bfloat16(), normal(21, rows, hidden).bfloat16(), normal(22, rows, 2, inter).bfloat16()
    dx, dgu, dd, dw = torch.zeros((rows, hidden), dtype=torch.bfloat16, device=DEV), torch.full_like(gate_up, 7.0), torch.full_like(down, 7.0), torch.zeros(rows, device=DEV)
    ctx.mw_ffn_backward(experts, x.to(DEV), offsets, kept.to(DEV), dy.to(DEV), dx, dgu, dd, ctx.ffn_workspace(experts, rows, True), None, dw)
    torch.cuda.synchronize()
    first = 0
    for e, c in counts.items():
        at = slice(first, first + c)
        first += c
        want = P.block_backward(host(x[at]), host(gate_up[e]), host(down[e]), np.ones(c), host(kept[at]), host(dy[at]))
        for got, (v, off), rounding in zip((dx[at], dgu[e], dd[e], dw[at]), want, (P.BF16,) * 3 + (P.U,)):
            near(got, v, off, rounding)
        dgu[e], dd[e] = 0, 0
    assert not dgu.any() and not dd.any()
