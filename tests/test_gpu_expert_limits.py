"""The experts' calls at the ends of what they take: rows MW_MAX_STRIDE elements apart, at every tile size, and MW_FFN_MAX_ROWS rows (exact_experts.py: results known to the bit)."""
import numpy as np
import pytest
import torch

import exact_experts as X
from paper_2605_22428_amd import binding as B
from test_gpu_expert_forms import Run, same, sevens

pytestmark = pytest.mark.gpu
DEV = X.DEV
# few rows; up of 256 x 128 and 256 x 256; down and dx of both; act of both; the large tiles of gradients
FAR = [X.CASES[1], X.CASES[5], X.CASES[7], X.CASES[9], X.CASES[11], X.CASES[15], X.CASES[16], X.CASES[19]]


def far(t, dtype=torch.bfloat16):
    """The rows of t, MW_MAX_STRIDE elements apart."""
    wide = torch.empty((t.shape[0] * B.MW_MAX_STRIDE,), dtype=dtype, device=DEV).view(t.shape[0], B.MW_MAX_STRIDE)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


@pytest.fixture(autouse=True, scope="module")
def _leave_no_cache():
    yield
    torch.cuda.empty_cache()


def _room(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < gib << 30:
        pytest.skip("%.0f GiB of device memory free, %d needed" % (free / 2 ** 30, gib))


@pytest.mark.parametrize("case", FAR)
def test_rows_far_apart(case):
    _room(40)
    r = Run(*case)
    b = r.b
    x, rows, dy, y, dx = far(b.x), far(b.rows), far(b.dy), far(torch.full_like(b.x, 7.0)), far(torch.full_like(b.x, 7.0))
    kept, dgu, dd, dw = sevens(b.room, 2, b.inter), sevens(*b.gate_up.shape), sevens(*b.down.shape), sevens(b.room, dtype=torch.float32)
    r.ctx.mw_ffn(r.experts, x, r.offsets, y, r.workspace(False), r.w, kept)
    r.ctx.mw_ffn_backward(r.experts, rows, r.offsets, r.kept, dy, dx, dgu, dd, r.workspace(True), r.w, dw)
    torch.cuda.synchronize()
    same((y, kept, dx, dgu, dd, dw), b.forward(X.few(case)) + b.backward())


@pytest.mark.parametrize("counts,n_in,n_out", [c for c in X.MATRIX_CASES if sum(c[0]) < 1000])
def test_codes_far_apart(counts, n_in, n_out):
    _room(8)
    codes, scales, w, w_scale, want = X.matrices(counts, n_in, n_out, spare=3)
    out = far(torch.full((codes.shape[0], n_out), 7.0), torch.float32)
    B.MatricesInt8(w, w_scale).mw_matmul_int8(far(codes, torch.int8), scales, X.offsets_of(counts, 0), out)
    torch.cuda.synchronize()
    same([out], [want])


def test_quantized_rows_far_apart():
    _room(8)
    x = torch.randn((300, 272), generator=torch.Generator(DEV).manual_seed(1), device=DEV).bfloat16()
    codes, scales = far(torch.full((300, 272), 99, dtype=torch.int8), torch.int8), torch.empty(300, device=DEV)
    B.mw_quantize_rows(far(x), codes, scales)
    torch.cuda.synchronize()
    want, want_scales = X.codes_of(x)
    same([codes, scales], [want.to(torch.int8), want_scales])


@pytest.mark.parametrize("n", [3, 2000])
def test_the_most_rows(n):
    """2^24 rows over three experts and over 2000."""
    _room(40)
    rows = B.MW_FFN_MAX_ROWS
    counts = [rows // n + (e % 2) * 5 for e in range(n - 1)]
    counts.append(rows - sum(counts))
    r = Run(counts, 16, 16)
    y, kept = r.forward()
    # in slices, as 64-bit forms of all rows at once take too much room
    for e, at in list(X.runs(counts, 0))[:: max(n // 7, 1)] + [list(X.runs(counts, 0))[-1]]:
        for first in (at.start, max(at.stop - 70000, at.start)):
            part = slice(first, min(first + 70000, at.stop))
            x, (gate, up) = r.b.x[part], r.b.gate_up[e]
            g, u = x @ gate.T, x @ up.T
            want = r.b.w[part, None].double() * ((g * u).bfloat16().double() @ r.b.down[e].T)
            same([y[part], kept[part]], [want.bfloat16(), torch.stack((g, u), 1).bfloat16()])
    with pytest.raises(B.MwError) as error:
        r.ctx.ffn_workspace(r.experts, rows + 1)
    assert error.value.status == B.MW_ERR_CAPACITY


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_the_largest_experts(rows):
    """gate_up of 2 GiB each, the second expert's rows: matrices hold whole numbers at their ends and zeros between, so results are known to the bit; zeros where zeros belong."""
    _room(40)
    hidden, inter = 16384, 32768
    g = torch.Generator(DEV).manual_seed(rows)
    whole = lambda *shape: torch.randint(-1, 2, shape, generator=g, device=DEV, dtype=torch.int8).bfloat16()
    rim = lambda n: torch.cat((torch.arange(300), torch.arange(n // 2 - 150, n // 2 + 150), torch.arange(n - 300, n))).to(DEV)
    at_h, at_i = rim(hidden), rim(inter)
    gate_up, down = torch.zeros((2, 2, inter, hidden), dtype=torch.bfloat16, device=DEV), torch.zeros((2, hidden, inter), dtype=torch.bfloat16, device=DEV)
    gate_up[:, 0, :, 0], gate_up[1, 1, at_i] = 4, whole(900, hidden)
    corner = whole(900, 900)
    down[1, at_h[:, None], at_i[None, :]] = corner
    x, dy, kept = whole(rows, hidden), whole(rows, hidden), torch.stack((torch.full((rows, inter), 32.0, device=DEV), whole(rows, inter).float()), 1).bfloat16()
    x[:, 0] = 8
    ctx = B.Context(1, 2, 1, 0, hidden, B.MW_ROW_BF16, 1, 1, np.zeros(2, dtype=np.int32))
    experts, offsets = B.Experts(gate_up, down), torch.tensor([0, 0, rows], device=DEV)
    assert 2 * gate_up[0].numel() == 2 << 30
    y, got_kept, dx, dw, ws = sevens(rows, hidden), sevens(rows, 2, inter), sevens(rows, hidden), sevens(rows, dtype=torch.float32), ctx.ffn_workspace(experts, rows, True)
    dgu, dd = torch.full_like(gate_up, 7.0), torch.full_like(down, 7.0)
    ctx.mw_ffn(experts, x, offsets, y, ws, None, got_kept)
    ctx.mw_ffn_backward(experts, x, offsets, kept, dy, dx, dgu, dd, ws, None, dw)
    torch.cuda.synchronize()
    u = x.double() @ gate_up[1, 1, at_i].double().T
    h = 32 * u
    high = h.bfloat16().double()
    h = high + (h - high).bfloat16().double() if rows <= 20 else high
    want = torch.zeros((rows, hidden), dtype=torch.float64, device=DEV)
    want[:, at_h] = h @ corner.double().T
    same([y], [want.bfloat16()])
    want_kept = torch.zeros((rows, 2, inter), dtype=torch.float64, device=DEV)
    want_kept[:, 0], want_kept[:, 1, at_i] = 32, u
    same([got_kept], [want_kept.bfloat16()])
    da, k = dy[:, at_h].double() @ corner.double(), kept[:, 1, at_i].double()
    d_gate, d_up = (da * k).bfloat16().double(), (da * 32).bfloat16().double()
    want = d_up @ gate_up[1, 1, at_i].double()
    want[:, 0] += 4 * d_gate.sum(1)
    same([dx, dw], [want.bfloat16(), (da * 32 * k).sum(1).float()])
    same([dgu[1, 0, at_i], dgu[1, 1, at_i]], [(d_gate.T @ x.double()).bfloat16(), (d_up.T @ x.double()).bfloat16()])
    dgu[1, :, at_i] = 0
    assert not dgu.any()
    for i in range(0, inter, 4096):
        same([dd[1, :, i:i + 4096]], [(dy.double().T @ (32 * kept[:, 1, i:i + 4096].double())).bfloat16()])
    assert not dd[0].any()
