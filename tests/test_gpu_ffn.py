"""mw_ffn and mw_ffn_backward against a plain 64-bit form (plain_experts.py derives how far they may be off)."""
import itertools

import numpy as np
import pytest
import torch

import plain_experts as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def host(t):
    return t.double().cpu().numpy()


def near(got, want, off, rounding=P.BF16):
    got = host(got)
    bad = ~(np.abs(got - want) <= off + rounding * (np.abs(want) + off) + 1e-30)
    assert not bad.any(), (bad.sum(), np.abs(got - want)[bad].max(), np.argwhere(bad)[:5])


class Set:
    """Experts with rows: counts[e] rows of expert e, `spare` rows of none behind them."""

    def __init__(self, counts, hidden, inter, spare=0, seed=1, weighted=True, pad=0):
        self.counts, self.hidden, self.inter, n = counts, hidden, inter, len(counts)
        self.rows, self.room = sum(counts), sum(counts) + spare
        self.gate_up, self.down = ((normal(seed + i, *s) * s[-1] ** -0.5).bfloat16() for i, s in enumerate(((n, 2, inter, hidden), (n, hidden, inter))))
        self.x, self.dy = (normal(seed + i, self.room, hidden).bfloat16() for i in (2, 3))
        self.kept = normal(seed + 4, self.room, 2, inter).bfloat16()
        self.w = torch.rand(self.room, generator=torch.Generator().manual_seed(seed)) * 2 - 0.5 if weighted else None
        for t in (self.x, self.dy, self.kept) + ((self.w,) if weighted else ()):
            t[self.rows:] = float("nan")                                  # rows of no expert
        self.offsets = torch.tensor([0] + list(itertools.accumulate(counts)), dtype=torch.int64, device=DEV)
        self.ctx = B.Context(1, max(n, 1), 1, 0, hidden, B.MW_ROW_BF16, 1, max(self.room, 1), np.zeros(max(n, 1), dtype=np.int32))
        self.dev = B.Experts(self.gate_up.to(DEV), self.down.to(DEV))
        self.dev_x, self.dev_dy, self.dev_kept = strided(self.x, pad), strided(self.dy, pad), self.kept.to(DEV)
        self.dev_w = self.w.to(DEV) if weighted else None
        self.pad = pad

    def workspace(self, backward):
        ws = self.ctx.ffn_workspace(self.dev, self.room, backward)
        ws.fill_(0xff)                                                    # (no part of it has to be prepared)
        return ws

    def forward(self, keep=True):
        y = torch.full((self.room, self.hidden + self.pad), 7.0, dtype=torch.bfloat16, device=DEV)
        kept = torch.full((self.room, 2, self.inter), 7.0, dtype=torch.bfloat16, device=DEV) if keep else None
        self.ctx.mw_ffn(self.dev, self.dev_x, self.offsets, y[:, :self.hidden], self.workspace(False), self.dev_w, kept)
        torch.cuda.synchronize()
        assert (y[self.rows:] == 7).all() and (y[:, self.hidden:] == 7).all() and (kept is None or (kept[self.rows:] == 7).all())
        return y[:self.rows, :self.hidden], None if kept is None else kept[:self.rows]

    def backward(self, **leave):
        dx = torch.full((self.room, self.hidden + self.pad), 7.0, dtype=torch.bfloat16, device=DEV)
        dgu, dd = (torch.full(t.shape, 7.0, dtype=torch.bfloat16, device=DEV) for t in (self.gate_up, self.down))
        dw = torch.full((self.room,), 7.0, device=DEV)
        out = [None if k in leave else t for k, t in (("dx", dx[:, :self.hidden]), ("dgu", dgu), ("dd", dd), ("dw", dw))]
        self.ctx.mw_ffn_backward(self.dev, self.dev_x, self.offsets, self.dev_kept, self.dev_dy, out[0], out[1], out[2], self.workspace(True), self.dev_w, out[3])
        torch.cuda.synchronize()
        assert (dx[self.rows:] == 7).all() and (dx[:, self.hidden:] == 7).all() and (dw[self.rows:] == 7).all()
        for k, t in (("dx", dx), ("dgu", dgu), ("dd", dd), ("dw", dw)):
            assert k not in leave or (t == 7).all()
        return dx[:self.rows, :self.hidden], dgu, dd, dw[:self.rows]

    def runs(self):
        first = 0
        for e, c in enumerate(self.counts):
            if c:
                yield e, slice(first, first + c), (np.ones(c) if self.w is None else host(self.w[first:first + c]))
            first += c

    def check_forward(self, keep=True):
        y, kept = self.forward(keep)
        for e, at, w in self.runs():
            (want, off), (want_kept, off_kept) = P.block(host(self.x[at]), host(self.gate_up[e]), host(self.down[e]), w)
            near(y[at], want, off)
            if keep:
                near(kept[at], want_kept, off_kept)

    def check_backward(self, **leave):
        dx, dgu, dd, dw = self.backward(**leave)
        hit = set()
        for e, at, w in self.runs():
            hit.add(e)
            want = P.block_backward(host(self.x[at]), host(self.gate_up[e]), host(self.down[e]), w, host(self.kept[at]), host(self.dy[at]))
            for k, got, (v, off), rounding in (("dx", dx[at], want[0], P.BF16), ("dgu", dgu[e], want[1], P.BF16), ("dd", dd[e], want[2], P.BF16), ("dw", dw[at], want[3], P.U)):
                if k not in leave:
                    near(got, v, off, rounding)
        for e in range(len(self.counts)):
            assert e in hit or "dgu" in leave or (dgu[e] == 0).all()
            assert e in hit or "dd" in leave or (dd[e] == 0).all()


# counts, hidden, inter: one row, few rows, rows that end a tile or begin one, experts without rows, sizes that are no multiples of a tile or a step
SIZES = [([1], 8, 8), ([1], 256, 264), ([0, 1, 0], 72, 136), ([3, 0, 5], 328, 72), ([16], 64, 64), ([17, 15, 1], 136, 200), ([33, 64, 65], 264, 328), ([31, 0, 127, 1], 128, 256),
         ([129], 520, 40), ([255], 200, 392), ([256], 256, 128), ([257, 200], 264, 136), ([600], 72, 520), ([300, 500, 0, 31], 328, 264), ([0, 0], 64, 64), ([700, 1, 2], 128, 64), ([400, 0, 300], 1032, 1048), ([20, 40], 1544, 2056), ([520], 2056, 264)]


@pytest.mark.parametrize("counts,hidden,inter", SIZES)
def test_forward(counts, hidden, inter):
    Set(counts, hidden, inter, spare=len(counts) % 3 * 5, pad=8 * (hidden % 3)).check_forward()
    Set(counts, hidden, inter, weighted=False, seed=9).check_forward(keep=False)


@pytest.mark.parametrize("counts,hidden,inter", SIZES)
def test_backward(counts, hidden, inter):
    Set(counts, hidden, inter, spare=len(counts) % 3 * 5, pad=8 * (hidden % 3)).check_backward()
    Set(counts, hidden, inter, weighted=False, seed=9).check_backward(dw=True)


@pytest.mark.parametrize("counts,hidden,inter", [([2, 1], 7168, 256), ([40], 1024, 2048), ([200, 57], 4096, 72)])
def test_long_sums(counts, hidden, inter):
    s = Set(counts, hidden, inter, spare=3)
    s.check_forward()
    s.check_backward()


def test_more_experts_than_a_wave_has_lanes():
    counts = [(7 * e) % 5 if e % 9 else 0 for e in range(150)]
    counts[70], counts[149] = 40, 3
    s = Set(counts, 64, 72, spare=2)
    s.check_forward()
    s.check_backward()


@pytest.mark.parametrize("n,runs", [(40, {3: 600, 39: 33}), (100, {80: 1200, 99: 17, 2: 16}), (70, {0: 33, 64: 1000, 65: 32}), (3, {1: 48}), (300, {5: 70, 250: 17, 299: 1}), (300, {299: 33})])
def test_few_rows_most_of_which_are_one_experts(n, runs):
    """At most sixteen rows an expert on average: the form of few rows, with runs of many."""
    counts = [runs.get(e, 0) for e in range(n)]
    assert sum(counts) + 3 <= 16 * n or n == 3
    Set(counts, 136, 72, spare=3 if n > 3 else 0, pad=8).check_forward()


@pytest.mark.parametrize("leave", [("dx",), ("dgu", "dd"), ("dx", "dgu", "dw"), ("dx", "dd", "dw")])
def test_gradients_that_are_left_out(leave):
    Set([70, 0, 20], 136, 72, spare=1).check_backward(**{k: True for k in leave})


def test_no_rows():
    s = Set([0, 0, 0], 64, 64)
    y, _ = s.forward()
    assert y.shape == (0, 64)
    dx, dgu, dd, dw = s.backward()
    assert (dgu == 0).all() and (dd == 0).all()


def test_a_rank_without_experts():
    ctx = B.Context(2, 1, 1, 0, 64, B.MW_ROW_BF16, 1, 4, np.ones(1, dtype=np.int32))
    experts = B.Experts(*(torch.empty(v, dtype=torch.bfloat16, device=DEV) for v in ((0, 2, 32, 64), (0, 64, 32))))
    x, y, offsets = normal(1, 4, 64).bfloat16().to(DEV), torch.full((4, 64), 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    ctx.mw_ffn(experts, x, offsets, y, ctx.ffn_workspace(experts, 4))
    kept = torch.zeros((4, 2, 32), dtype=torch.bfloat16, device=DEV)
    ctx.mw_ffn_backward(experts, x, offsets, kept, x, y, experts._held[0], experts._held[1], ctx.ffn_workspace(experts, 4, True))
    torch.cuda.synchronize()
    assert (y == 7).all()


@pytest.mark.parametrize("rows", [3, 70, 300])
def test_values_that_are_not_finite_stay_in_their_rows(rows):
    """An infinity or a NaN in one expert's rows reaches neither other rows nor other experts' gradients."""
    clean, s = (Set([rows, rows, rows], 136, 72, seed=3) for _ in range(2))
    bad = rows + rows // 2
    for t, v in ((s.dev_x, float("nan")), (s.dev_dy, float("inf"))):
        t[bad, 5] = v
    (y, kept), (want, want_kept) = s.forward(), clean.forward()
    others = [r for r in range(3 * rows) if r != bad]
    assert torch.equal(y[others], want[others]) and torch.equal(kept[others], want_kept[others]) and y[bad].isnan().all()
    got, want = s.backward(), clean.backward()
    for k in (0, 3):
        assert torch.equal(got[k][others], want[k][others])
    for k in (1, 2):
        assert torch.equal(got[k][[0, 2]], want[k][[0, 2]]) and not got[k][1].isfinite().all()


def test_gates_far_from_zero():
    """silu of values whose exponential over- or underflows."""
    s = Set([20], 64, 64)
    s.dev_kept[:, 0] = torch.tensor([-3e38, -1000.0, -104.0, -88.0, 0.0, 88.0, 1000.0, 3e38], device=DEV).repeat(8).bfloat16()
    s.kept = s.dev_kept.cpu()
    dx, dgu, dd, dw = s.backward()
    g = host(s.kept[:20, 0])
    assert dgu[0, 0][:, :].isfinite().all() and (dgu[0, 1][g[0] <= -1000] == 0).all() and (dd[0][:, g[0] <= -1000] == 0).all()
    s.kept[:, 0] = s.kept[:, 0].clamp(-100, 100)
    s.dev_kept.copy_(s.kept)
    s.check_backward()


def test_offsets_outside_the_rows_count_as_the_nearest_inside():
    s = Set([4, 5, 6], 64, 72)
    want, _ = s.forward()
    s.offsets.copy_(torch.tensor([-3, 4, 9, 1 << 40]))
    got, _ = s.forward()
    assert torch.equal(got, want)
    first = s.backward()
    s.offsets.copy_(torch.tensor([0, 4, 9, 15]))
    assert all(torch.equal(a, b) for a, b in zip(first, s.backward()))


@pytest.mark.parametrize("before,counts", [(3, [4, 5]), (40, [70, 0, 30]), (300, [300, 200])])
def test_rows_before_the_first_expert_are_left_as_they_were(before, counts):
    """The same rows behind `before` rows of no expert give the same values, and those rows are neither read nor written.  (Experts with as many rows: the
    room's size may choose other tiles, so values are held against the plain form.)"""
    s = Set([before] + counts, 136, 72, spare=2)
    s.offsets[0] = before                                                 # the first expert's rows are no expert's now
    s.counts[0] = 0
    s.offsets[1] = before
    for t in (s.x, s.dy, s.kept, s.w):
        t[:before] = float("nan")
    s.dev_x[:before], s.dev_dy[:before], s.dev_kept[:before], s.dev_w[:before] = (float("nan"),) * 4
    y, kept = s.forward()
    dx, dgu, dd, dw = s.backward()
    assert all((t[:before] == 7).all() for t in (y, kept, dx, dw)) and (dgu[0] == 0).all() and (dd[0] == 0).all()
    first = before
    for e, c in list(enumerate(counts, 1)):
        if c:
            at, w = slice(first, first + c), host(s.w[first:first + c])
            (want, off), _ = P.block(host(s.x[at]), host(s.gate_up[e]), host(s.down[e]), w)
            near(y[at], want, off)
            want = P.block_backward(host(s.x[at]), host(s.gate_up[e]), host(s.down[e]), w, host(s.kept[at]), host(s.dy[at]))
            for got, (v, off), rounding in ((dx[at], want[0], P.BF16), (dgu[e], want[1], P.BF16), (dd[e], want[2], P.BF16), (dw[at], want[3], P.U)):
                near(got, v, off, rounding)
        first += c


def test_gradients_against_differences():
    """L = sum of dy y; central differences of a 64-bit forward pass in random directions of x, weights and gate weights.  The step is 2^-12 of a
    direction of the values' own size: the difference is off by 2^-24 times L's cubic term along it, which is below 100 sizes of the gradient's product here; the gradient by its
    roundings, 2^-8 for each of three places, at random signs: their sum over N values stays below 6 sqrt(sum of squares) times that."""
    s = Set([9, 0, 30], 48, 40, seed=5)
    _, kept = s.forward()
    s.dev_kept[:s.rows] = kept
    grads = s.backward()

    def value(x, gate_up, down, w):
        total = 0.0
        for e, at, _ in s.runs():
            g, u = x[at] @ gate_up[e, 0].T, x[at] @ gate_up[e, 1].T
            total += (w[at, None] * ((g * P.sig(g) * u) @ down[e].T) * host(s.dy[at])).sum()
        return total

    start = [host(s.x), host(s.gate_up), host(s.down), host(s.w)]
    for k, grad in enumerate(grads):
        d = host(normal(50 + k, *start[k].shape)) * np.abs(start[k])
        ends = [value(*[v + sign * 2.0 ** -12 * d if i == k else v for i, v in enumerate(start)]) for sign in (1, -1)]
        along = host(grad) * d
        slack = 3 * P.BF16 * 6 * np.sqrt((along ** 2).sum()) + 2.0 ** -24 * 100 * np.abs(along).sum()
        assert abs((ends[0] - ends[1]) * 2.0 ** 11 - along.sum()) <= slack, (k, slack)


@pytest.mark.parametrize("counts", [[5, 9], [300, 400]])
def test_equal_calls_give_equal_bits(counts):
    s = Set(counts, 264, 200)
    first = s.forward() + s.backward()
    for _ in range(3):
        for u, v in zip(first, s.forward() + s.backward()):
            assert torch.equal(u, v)


@pytest.mark.parametrize("counts", [[2, 0, 3], [40, 60, 0], [300, 250, 90]])
def test_replayed_from_a_graph_on_another_stream(counts):
    """A step of forward and backward, captured, with other rows, counts and weights before every replay."""
    s = Set(counts, 136, 72, spare=4)
    y, kept = torch.empty((s.room, 136), dtype=torch.bfloat16, device=DEV), torch.empty((s.room, 2, 72), dtype=torch.bfloat16, device=DEV)
    dx, dgu, dd, dw = torch.empty_like(y), torch.empty_like(s.dev._held[0]), torch.empty_like(s.dev._held[1]), torch.empty(s.room, device=DEV)
    x, dy, w, ws = torch.zeros_like(y), torch.zeros_like(y), torch.zeros(s.room, device=DEV), s.workspace(True)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step():
        s.ctx.mw_ffn(s.dev, x, s.offsets, y, ws, w, kept)
        s.ctx.mw_ffn_backward(s.dev, x, s.offsets, kept, dy, dx, dgu, dd, ws, w, dw)

    with torch.cuda.stream(st):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
    for seed in range(4):
        s.counts = list(np.roll(counts, seed))
        s.offsets.copy_(torch.tensor([0] + list(itertools.accumulate(s.counts))))
        s.x, s.dy, s.w = normal(20 + seed, s.room, 136).bfloat16(), normal(30 + seed, s.room, 136).bfloat16(), normal(40 + seed, s.room)
        for to, v in ((x, s.x), (dy, s.dy), (w, s.w)):
            to.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for e, at, wt in s.runs():
            (want, off), (want_kept, off_kept) = P.block(host(s.x[at]), host(s.gate_up[e]), host(s.down[e]), wt)
            near(y[at], want, off)
            near(kept[at], want_kept, off_kept)
            for got, (v, off), r in zip((dx[at], dgu[e], dd[e], dw[at]),
                                        P.block_backward(host(s.x[at]), host(s.gate_up[e]), host(s.down[e]), wt, host(kept[at]), host(s.dy[at])), (P.BF16,) * 3 + (P.U,)):
                near(got, v, off, r)
        eager = [t.clone() for t in (y, kept, dx, dgu, dd, dw)]
        step()
        torch.cuda.synchronize()
        n = sum(s.counts)
        for a, b in zip(eager, (y, kept, dx, dgu, dd, dw)):
            assert torch.equal(a[:n] if a.shape[0] == s.room else a, b[:n] if b.shape[0] == s.room else b)


def _step(s, out, ws):
    y, kept, dx, dgu, dd, dw = out
    s.ctx.mw_ffn(s.dev, s.dev_x, s.offsets, y, ws, s.dev_w, kept)
    s.ctx.mw_ffn_backward(s.dev, s.dev_x, s.offsets, kept, s.dev_dy, dx, dgu, dd, ws, s.dev_w, dw)


def _outputs(s):
    return ([torch.zeros((s.room, s.hidden), dtype=torch.bfloat16, device=DEV), torch.zeros((s.room, 2, s.inter), dtype=torch.bfloat16, device=DEV), torch.zeros((s.room, s.hidden), dtype=torch.bfloat16, device=DEV)] +
            [torch.zeros_like(t) for t in s.dev._held[:2]] + [torch.zeros(s.room, device=DEV)])


@pytest.mark.parametrize("counts", [[9, 3], [200, 130], [700, 300]])
def test_calls_on_two_streams_at_once(counts):
    """Two contexts' steps side by side, each with its own workspace and stream, give what they give alone."""
    sets = [Set(counts, 264, 328, seed=1), Set(counts[::-1], 264, 328, seed=50)]
    want = [_outputs(s) for s in sets]
    for s, o in zip(sets, want):
        _step(s, o, s.workspace(True))
        torch.cuda.synchronize()
    got, spaces, streams = [_outputs(s) for s in sets], [s.workspace(True) for s in sets], [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(6):
        for s, o, ws, st in zip(sets, got, spaces, streams):
            with torch.cuda.stream(st):
                _step(s, o, ws)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("counts", [[9, 3], [200, 130]])
def test_two_graphs_that_share_a_workspace(counts):
    """Replayed in turn, with the eager step between them, each finds nothing in the workspace that it needs and leaves nothing that the other minds."""
    sets = [Set(counts, 264, 328, seed=1), Set([c + 40 for c in counts], 264, 328, seed=50)]
    want, got, graphs = [_outputs(s) for s in sets], [_outputs(s) for s in sets], []
    ws = sets[1].workspace(True)                                          # (the larger one)
    for s, o in zip(sets, want):
        _step(s, o, ws)
        torch.cuda.synchronize()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for s, o in zip(sets, got):
        with torch.cuda.stream(st):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                _step(s, o, ws)
        graphs.append(graph)
    for turn in (0, 1, 0, 0, 1, 1, 0):
        for t in got[turn]:
            t.zero_()
        ws.fill_(turn * 77)
        torch.cuda.synchronize()
        graphs[turn].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want[turn], got[turn]))
        _step(sets[1 - turn], _outputs(sets[1 - turn]), ws)


def test_refusals():
    s = Set([3, 2], 64, 32)
    I, CAP, WS, UN = B.MW_ERR_INVALID_ARG, B.MW_ERR_CAPACITY, B.MW_ERR_WORKSPACE, B.MW_ERR_UNSUPPORTED
    y, odd = torch.empty((5, 64), dtype=torch.bfloat16, device=DEV), torch.zeros(4096, dtype=torch.bfloat16, device=DEV)
    ws, h = s.workspace(True), s.ctx._h
    call, good = B._native().mw_ffn, [h, s.dev.address, s.dev_x, 64, s.offsets, 5, s.dev_w, y, 64, s.dev_kept, ws, ws.numel(), 0]
    assert call(*good) == B.MW_OK
    for at, bad, status in ((0, None, I), (1, 0, I), (2, None, I), (2, odd[4:], I), (3, 56, I), (3, 68, I), (3, (1 << 21) + 8, UN), (4, None, I), (5, -1, I), (5, (1 << 24) + 1, CAP),
                            (6, odd[1:], I), (7, None, I), (7, odd[1:], I), (8, 60, I), (8, 1 << 22, UN), (9, odd[4:], I), (10, None, WS), (10, ws[8:], WS), (11, 100, WS)):
        assert call(*(good[:at] + [bad] + good[at + 1:])) == status, (at, bad)
    dgu, dd, dw = torch.empty_like(s.dev._held[0]), torch.empty_like(s.dev._held[1]), torch.empty(5, device=DEV)
    back, good_b = B._native().mw_ffn_backward, [h, s.dev.address, s.dev_x, 64, s.offsets, 5, s.dev_w, s.dev_kept, s.dev_dy, 64, y, 64, dgu, dd, dw, ws, ws.numel(), 0]
    assert back(*good_b) == B.MW_OK
    for at, bad, status in ((0, None, I), (1, 0, I), (2, None, I), (3, 56, I), (3, 1 << 22, UN), (4, None, I), (5, -1, I), (5, (1 << 24) + 1, CAP), (7, None, I), (7, odd[4:], I), (8, None, I), (9, 36, I),
                            (9, 1 << 22, UN), (10, odd[1:], I), (11, 12, I), (11, 1 << 22, UN), (12, odd[1:], I), (13, odd[1:], I), (14, odd[1:], I), (15, None, WS), (16, 64, WS)):
        assert back(*(good_b[:at] + [bad] + good_b[at + 1:])) == status, (at, bad)
    for change, status in ((dict(inter=0), I), (dict(inter=28), UN), (dict(format=7), I), (dict(format=B.MW_ROW_FP8_E4M3_BLOCK128), UN), (dict(gate_up_dev=0), I), (dict(down_dev=s.dev.record.down_dev + 2), I),
                           (dict(down_scale_dev=s.dev.record.down_dev), I), (dict(inter=1 << 24), UN)):
        rec = B.MwExperts(*[change.get(f, getattr(s.dev.record, f)) for f, _ in B.MwExperts._fields_])
        assert call(*([h, B.C.addressof(rec)] + good[2:])) == status, change
        assert back(*([h, B.C.addressof(rec)] + good_b[2:])) == status, change
    with pytest.raises(B.MwError) as e:
        s.ctx.ffn_workspace(s.dev, (1 << 24) + 1)
    assert e.value.status == CAP
    other = B.Experts(*(torch.zeros(v, dtype=torch.bfloat16, device=DEV) for v in ((1, 2, 32, 64), (1, 64, 32))))
    for args in ((other, s.dev_x, s.offsets, y, ws), (s.dev, s.dev_x.float(), s.offsets, y, ws), (s.dev, s.dev_x, s.offsets.int(), y, ws), (s.dev, s.dev_x, s.offsets[:2], y, ws),
                 (s.dev, s.dev_x, s.offsets, y[:4], ws), (s.dev, s.dev_x[:, ::2], s.offsets, y, ws), (s.dev, s.dev_x, s.offsets, y, ws, dw[:4]), (s.dev, s.dev_x, s.offsets, y, ws, None, s.dev_kept[:, :1])):
        with pytest.raises(ValueError):
            s.ctx.mw_ffn(*args)
    with pytest.raises(ValueError):
        s.ctx.mw_ffn_backward(s.dev, s.dev_x, s.offsets, s.dev_kept, s.dev_dy, y, dgu[:1], dd, ws)
