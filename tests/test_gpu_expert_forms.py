"""Every tile size of the experts' products and of their gradients, with whole tiles and tiles in parts (test_expert_forms.py holds that these sizes reach them), on whole numbers whose
results are known to the bit (exact_experts.py); what surrounds a product (rows of no expert, values that are not finite, graphs, streams) at the larger tiles too."""
import numpy as np
import pytest
import torch

import exact_experts as X
from paper_2605_22428_amd import binding as B
from test_gpu_ffn import Set, _outputs, _step

pytestmark = pytest.mark.gpu
DEV = X.DEV
NAMES = ["-".join(map(str, c[0])) + "_%dx%d" % c[1:3] for c in X.CASES]
# a size for each pair of forms of the larger tiles: up, down, act and dx of 256 x 128 and of 256 x 256, whole and in parts, and both sizes of gradients
LARGER = [([513, 0, 589], 4104, 328, 1, 0), ([257, 0, 143], 8200, 72, 4, 0), ([257, 0, 1, 300, 142], 8200, 72, 0, 2), ([140, 0, 260], 72, 8200, 9, 0), ([2301, 0, 1707], 8200, 136, 0, 5), ([3003, 1001], 264, 8200, 3, 0)]


def padded(t, pad):
    """t with `pad` columns of NaN behind each row, bf16."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def sevens(*shape, dtype=torch.bfloat16):
    return torch.full(shape, 7.0, dtype=dtype, device=DEV)


class Run:
    def __init__(self, counts, hidden, inter, before=0, spare=0, pad=0, seed=1):
        self.b = b = X.Block(counts, hidden, inter, before, spare, seed)
        self.pad, n = pad, len(counts)
        self.ctx = B.Context(1, n, 1, 0, hidden, B.MW_ROW_BF16, 1, 1, np.zeros(n, dtype=np.int32))
        self.experts = B.Experts(b.gate_up.bfloat16(), b.down.bfloat16())
        self.offsets = X.offsets_of(counts, before)
        self.x, self.rows, self.dy = padded(b.x, pad), padded(b.rows, pad), padded(b.dy, pad)
        self.kept, self.w = b.kept.bfloat16(), b.w.float()

    def workspace(self, backward):
        ws = self.ctx.ffn_workspace(self.experts, self.b.room, backward)
        return ws.fill_(0xff)

    def forward(self):
        b, y = self.b, sevens(self.b.room, self.b.hidden + self.pad)
        kept = sevens(b.room, 2, b.inter)
        self.ctx.mw_ffn(self.experts, self.x, self.offsets, y[:, :b.hidden], self.workspace(False), self.w, kept)
        torch.cuda.synchronize()
        assert (y[:, b.hidden:] == 7).all()
        return y[:, :b.hidden], kept

    def backward(self, dx=True, matrices=True, dw=True):
        b, out = self.b, sevens(self.b.room, self.b.hidden + self.pad)
        got = [out[:, :b.hidden] if dx else None] + [sevens(*t.shape) if matrices else None for t in (b.gate_up, b.down)] + [sevens(b.room, dtype=torch.float32) if dw else None]
        self.ctx.mw_ffn_backward(self.experts, self.rows, self.offsets, self.kept, self.dy, *got[:3], self.workspace(True), self.w, got[3])
        torch.cuda.synchronize()
        assert (out[:, b.hidden:] == 7).all()
        return got


def same(got, want):
    for i, (a, b) in enumerate(zip(got, want)):
        if a is not None:
            assert torch.equal(a, b), (i, int((a != b).sum()), (a != b).nonzero()[:4].tolist(), a[a != b][:4].tolist(), b[a != b][:4].tolist())


@pytest.mark.parametrize("case", X.CASES, ids=NAMES)
def test_forward(case):
    r = Run(*case, pad=8 * (case[1] % 5))
    same(r.forward(), r.b.forward(X.few(case)))


@pytest.mark.parametrize("case", X.CASES, ids=NAMES)
def test_backward(case):
    r = Run(*case, pad=8 * (case[1] % 5))
    same(r.backward(), r.b.backward())


@pytest.mark.parametrize("case", [X.CASES[2]] + LARGER[2:])
def test_gradients_one_by_one(case):
    """Rows' weights alone have a launch of their own; matrices' gradients without rows'; rows' alone."""
    r = Run(*case)
    want = r.b.backward()
    for leave in (dict(dx=False, matrices=False), dict(dx=False, dw=False), dict(matrices=False, dw=False)):
        same(r.backward(**leave), want)


@pytest.mark.parametrize("case", X.CODE_CASES, ids=lambda c: "-".join(map(str, c[0])) + "_%dx%d" % c[1:3])
def test_experts_of_codes(case):
    b = X.CodeBlock(*case)
    ctx = B.Context(1, b.n, 1, 0, b.hidden, B.MW_ROW_BF16, 1, max(b.room, 1), np.zeros(b.n, dtype=np.int32))
    experts = B.Experts(b.gate_up, b.down, b.gate_up_scale, b.down_scale)
    for weighted in (True, False):
        y, ws = sevens(b.room, b.hidden + 8), ctx.ffn_workspace(experts, b.room).fill_(0xff)
        ctx.mw_ffn(experts, padded(b.x, 16), X.offsets_of(b.counts, b.before), y[:, :b.hidden], ws, b.w if weighted else None)
        torch.cuda.synchronize()
        assert (y[:, b.hidden:] == 7).all()
        same([y[:, :b.hidden]], [b.forward(weighted)])


@pytest.mark.parametrize("case", X.CODE_CASES[3:])
def test_experts_of_codes_replayed_from_a_graph(case):
    """Other rows and runs before every replay, one row of them infinite: it is NaN and no other row minds."""
    counts, hidden, inter, before, spare = case
    b = X.CodeBlock(*case)
    ctx = B.Context(1, b.n, 1, 0, hidden, B.MW_ROW_BF16, 1, max(b.room, 1), np.zeros(b.n, dtype=np.int32))
    experts = B.Experts(b.gate_up, b.down, b.gate_up_scale, b.down_scale)
    x, offsets, y, ws, w, st = b.x.clone(), X.offsets_of(counts, before), sevens(b.room, hidden), ctx.ffn_workspace(experts, b.room), b.w.clone(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        ctx.mw_ffn(experts, x, offsets, y, ws, w)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.mw_ffn(experts, x, offsets, y, ws, w)
    for turn in range(3):
        other = X.CodeBlock(list(np.roll(counts, turn)), hidden, inter, before, spare, seed=20 + turn)
        want = other.forward()
        bad = before + sum(counts) // 2
        other.x[bad, 3], want[bad] = float("inf"), 9.0
        for to, v in ((x, other.x), (w, other.w), (offsets, X.offsets_of(other.counts, before))) + tuple(zip(experts._held, (other.gate_up, other.down, other.gate_up_scale, other.down_scale))):
            to.copy_(v)
        for again in (graph.replay, lambda: ctx.mw_ffn(experts, x, offsets, y, ws, w)):
            y.fill_(7.0)
            ws.fill_(turn * 85)
            torch.cuda.synchronize()
            again()
            torch.cuda.synchronize()
            assert y[bad].isnan().all()
            y[bad] = 9.0
            same([y], [want])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts,n_in,n_out", X.MATRIX_CASES)
def test_products_of_codes(counts, n_in, n_out, dtype):
    codes, scales, w, w_scale, want = X.matrices(counts, n_in, n_out, spare=3)
    wide = torch.full((codes.shape[0], n_in + 16), 99, dtype=torch.int8, device=DEV)
    wide[:, :n_in] = codes
    out = sevens(codes.shape[0], n_out + 8, dtype=dtype)
    B.MatricesInt8(w, w_scale).mw_matmul_int8(wide[:, :n_in], scales, X.offsets_of(counts, 0), out[:, :n_out])
    torch.cuda.synchronize()
    assert (out[:, n_out:] == 7).all()
    same([out[:, :n_out]], [want.to(dtype)])


@pytest.mark.parametrize("case", LARGER)
def test_values_that_are_not_finite_stay_in_their_rows(case):
    """A NaN or an infinity in a row of the last expert reaches no other row and no other expert's gradients."""
    r = Run(*case, pad=8)
    b = r.b
    (y, kept), want = r.forward(), r.b.forward(X.few(case))
    back = r.b.backward()
    bad, last = b.before + sum(b.counts) - 2, max(e for e, c in enumerate(b.counts) if c)
    r.x[bad, 5], r.dy[bad, 6], r.rows[bad, 7] = float("nan"), float("inf"), float("nan")
    others = [i for i in range(b.room) if i != bad]
    y, kept = r.forward()
    same([y[others], kept[others]], [want[0][others], want[1][others]])
    assert y[bad].isnan().all()
    dx, dgu, dd, dw = r.backward()
    same([dx[others], dw[others]], [back[0][others], back[3][others]])
    experts = [e for e in range(b.n) if e != last]
    same([dgu[experts], dd[experts]], [back[1][experts], back[2][experts]])
    assert not dgu[last].isfinite().all() and not dd[last].isfinite().all()


@pytest.mark.parametrize("case", LARGER)
def test_replayed_from_a_graph_on_another_stream(case):
    """A step captured once; rows, weights and the runs' lengths change before every replay, an eager step stands between replays, the workspace holds anything."""
    counts, hidden, inter, before, spare = case
    r = Run(*case)
    room, ws, st = r.b.room, r.workspace(True), torch.cuda.Stream()
    y, kept, dx, dw = sevens(room, hidden), sevens(room, 2, inter), sevens(room, hidden), sevens(room, dtype=torch.float32)
    dgu, dd = sevens(*r.b.gate_up.shape), sevens(*r.b.down.shape)

    def step():
        r.ctx.mw_ffn(r.experts, r.x, r.offsets, y, ws, r.w, kept)
        r.ctx.mw_ffn_backward(r.experts, r.rows, r.offsets, r.kept, r.dy, dx, dgu, dd, ws, r.w, dw)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
    for turn in range(3):
        other = X.Block(list(np.roll(counts, turn)), hidden, inter, before, spare, seed=20 + turn)
        for to, v in ((r.x, other.x), (r.rows, other.rows), (r.dy, other.dy), (r.kept, other.kept), (r.w, other.w), (r.experts._held[0], other.gate_up), (r.experts._held[1], other.down),
                      (r.offsets, X.offsets_of(other.counts, before))):
            to.copy_(v)
        for t in (y, kept, dx, dw):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, want = (y, kept, dx, dgu, dd, dw), other.forward(X.few(case)) + other.backward()
        same(got, want)
        ws.fill_(turn)
        step()
        torch.cuda.synchronize()
        same(got, want)


@pytest.mark.parametrize("cases", [(0, 4), (2, 5), (1, 3)])
def test_calls_on_two_streams_at_once(cases):
    both = [Run(*LARGER[i], seed=30 + i) for i in cases]
    want = [r.b.forward(X.few(LARGER[i])) + r.b.backward() for i, r in zip(cases, both)]
    streams, spaces, outs = [torch.cuda.Stream() for _ in both], [r.workspace(True) for r in both], []
    for r in both:
        b = r.b
        outs.append((sevens(b.room, b.hidden), sevens(b.room, 2, b.inter), sevens(b.room, b.hidden), sevens(*b.gate_up.shape), sevens(*b.down.shape), sevens(b.room, dtype=torch.float32)))
    torch.cuda.synchronize()
    for _ in range(4):
        for r, st, ws, (y, kept, dx, dgu, dd, dw) in zip(both, streams, spaces, outs):
            with torch.cuda.stream(st):
                r.ctx.mw_ffn(r.experts, r.x, r.offsets, y, ws, r.w, kept)
                r.ctx.mw_ffn_backward(r.experts, r.rows, r.offsets, r.kept, r.dy, dx, dgu, dd, ws, r.w, dw)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        same(o, w)


@pytest.mark.parametrize("case", LARGER)
def test_values_of_all_sizes(case):
    """Normal values against the plain form, with what it may be off; equal calls give equal bits."""
    counts, hidden, inter, _, spare = case
    s = Set(counts, hidden, inter, spare=spare, pad=8)
    s.check_forward()
    s.check_backward()
    out = [_outputs(s) for _ in range(3)]
    ws = s.workspace(True)
    for o in out:
        _step(s, o, ws)
        torch.cuda.synchronize()
    for o in out[1:]:
        assert all(torch.equal(a[:s.rows] if a.shape[0] == s.room else a, b[:s.rows] if b.shape[0] == s.room else b) for a, b in zip(out[0], o))
