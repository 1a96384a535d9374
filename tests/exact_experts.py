"""Experts, rows and gradients of whole numbers, chosen so that every sum is exact in single precision and every rounding is known: results are compared for equality, and a term that is
lost, doubled or at another place shows whatever the length of its sum.

Gates are 18 or more, where 1 + exp(-g) is 1 in single precision and silu(g) is g.  Values are whole (with a row's weight whole or half), and the sizes of the terms of every sum add up to
less than 2^24, so any order gives the same.  Results in 64 bits are on the GPU.
CASES and the lists behind it: the sizes that are run."""
import itertools
import math

import torch

import tile_rules

DEV = "cuda:0"
FEW, SMALL, MIDDLE, LARGE = range(4)
TILE = {SMALL: (128, 64, 512), MIDDLE: (256, 128, 256), LARGE: (256, 256, 256)}          # columns, rows, tiles that run at a time

# counts, hidden, inter, rows before the first expert's, rows behind the last one's
CASES = [([5, 0, 9], 1096, 264, 2, 3), ([1, 0, 30, 0], 328, 136, 0, 1), ([130, 0, 69], 1544, 72, 0, 1), ([70, 131], 72, 1544, 3, 0), ([40, 160], 72, 776, 0, 0), ([129, 0, 67], 72, 8200, 0, 4),
         ([513, 0, 589], 4104, 328, 1, 0), ([130, 3, 171], 72, 8200, 2, 1), ([2301, 0, 1707], 8200, 136, 0, 5), ([257, 0, 143], 8200, 72, 4, 0), ([2605], 136, 8200, 0, 7), ([257, 0, 1, 300, 142], 8200, 72, 0, 2),
         ([3003, 1001], 264, 8200, 3, 0), ([4011], 8200, 264, 0, 0), ([1303, 1301], 8200, 136, 5, 0), ([255, 3, 0, 300, 145], 72, 8200, 0, 0), ([140, 0, 260], 72, 8200, 9, 0), ([1303, 0], 136, 8200, 0, 3),
         ([4003], 264, 4104, 0, 0), ([1000, 0, 601], 136, 8200, 0, 2)]
# experts of codes
CODE_CASES = [([5, 0, 9], 1104, 272, 2, 3), ([200, 0], 4112, 144, 0, 1), ([90, 111], 144, 4112, 3, 0), ([201], 144, 8208, 0, 2), ([130, 0, 171], 144, 8208, 1, 0), ([1103], 16400, 272, 0, 3), ([2203, 0, 1801], 16400, 144, 0, 0), ([4003], 16400, 144, 0, 1),
              ([1303], 144, 32784, 2, 0), ([257, 0, 147], 8208, 80, 0, 1), ([129, 1, 173], 16400, 144, 0, 0), ([3001, 1003], 272, 16400, 0, 4)]
# products of codes: counts, n_in, n_out
MATRIX_CASES = [([3, 0, 14], 272, 1040), ([70, 0, 131], 400, 272), ([129, 0, 67], 144, 16400), ([130, 3, 171], 2064, 16400), ([201], 2064, 16400), ([1000, 0, 3001], 144, 8208), ([33, 40], 8208, 80)]


def _products(counts, hidden, inter, before, spare, unit=64):
    """Of a case: name -> (columns, tile's share of columns, steps)."""
    one = {"up": (2 * inter, hidden), "down": (hidden, inter)}
    if unit == 64:
        one.update({"act": (inter, hidden), "dx": (hidden, 2 * inter)})
    return {k: (columns, -(-sums // unit)) for k, (columns, sums) in one.items()}


def forms(cases, unit=64):
    """For every case: product -> (form, parts of a tile of its last round, 0: no parts), and whether its matrices' gradients take the large tiles."""
    rooms = [sum(c[0]) + c[3] + c[4] for c in cases]
    ask = []
    for (counts, hidden, inter, *_), room in zip(cases, rooms):
        at = "(%d, %d, %d, %d)" % (room, len(counts), hidden, inter)
        if unit == 64:
            ask += ["forward_forms%s.first" % at, "forward_forms%s.second" % at, "backward_forms%s.first" % at, "backward_forms%s.second" % at, "grads_large%s" % at]
        else:
            ask += ["int8_form(%d, %d, %d, %d, true)" % (room, len(counts), 2 * inter, hidden), "int8_form(%d, %d, %d, %d, true)" % (room, len(counts), hidden, inter)]
    each = len(ask) // len(cases)
    got = tile_rules.values(("mw_few.h",), tuple(ask))
    ask, found = [], []
    for i, (case, room) in enumerate(zip(cases, rooms)):
        products = _products(*case, unit=unit)
        chosen = dict(zip(products, got[i * each:]))
        for k, (columns, steps) in products.items():
            if chosen[k] == FEW and k in ("act", "dx"):
                chosen[k] = SMALL
            if chosen[k] != FEW:
                p, q, round_ = TILE[chosen[k]]
                across = -(-columns // p)
                ask.append("split_tiles(%d, %d, %d, may_have_parts(%d, %d, %d, %d, %d)).parts" % (across * sum(-(-c // q) for c in case[0]), round_, steps, room, len(case[0]), q, across, steps))
        found.append((chosen, bool(got[i * each + 4]) if unit == 64 else False))
    parts = iter(tile_rules.values(("mw_few.h",), tuple(ask)))
    return [({k: (f, 0 if f == FEW else next(parts)) for k, f in chosen.items()}, grads) for chosen, grads in found]


def few(case):
    """Whether a case of CASES takes the form of few rows, which holds h as two bf16 values."""
    return sum(case[0]) + case[3] + case[4] <= 10 * len(case[0])


def _generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _whole(g, shape, most=1, density=1.0):
    v = torch.randint(-most, most + 1, shape, generator=g, device=DEV)
    return (v * (torch.rand(shape, generator=g, device=DEV) < density) if density < 1 else v).double()


def _weights(g, n):
    return torch.tensor([1.0, 2.0, -1.0, 0.5], device=DEV)[torch.randint(0, 4, (n,), generator=g, device=DEV)]


def _small(v, what):
    """Sums whose terms' sizes add up to this are exact in single precision in any order (terms are whole or halves)."""
    assert v.numel() == 0 or float(v.max()) < 2 ** 23, what
    return v


def _bf16(v):
    return v.bfloat16().double()


def offsets_of(counts, before):
    return torch.tensor([before] + [before + c for c in itertools.accumulate(counts)], dtype=torch.int64, device=DEV)


def runs(counts, before):
    first = before
    for e, c in enumerate(counts):
        if c:
            yield e, slice(first, first + c)
        first += c


class Block:
    """Inputs of mw_ffn and mw_ffn_backward in bf16 and what they give.  Rows of no expert are NaN."""

    def __init__(self, counts, hidden, inter, before=0, spare=0, seed=1):
        g = _generator(seed)
        self.counts, self.hidden, self.inter, self.before, self.n = counts, hidden, inter, before, len(counts)
        self.room = before + sum(counts) + spare
        self.gate_up = _whole(g, (self.n, 2, inter, hidden))
        self.gate_up[:, 0, :, 0] = math.ceil((18 + 6.5 * (0.45 * hidden) ** 0.5) / 8)          # (six deviations of the other terms' sum above 18)
        self.down = _whole(g, (self.n, hidden, inter))
        self.x, self.w = _whole(g, (self.room, hidden)), _weights(g, self.room)
        self.x[:, 0] = 8
        # the backward pass's own: rows, and g and u that a forward pass may have kept
        self.rows, self.dy = _whole(g, (self.room, hidden)), _whole(g, (self.room, hidden), density=0.5)
        self.kept = torch.stack((torch.randint(20, 41, (self.room, inter), generator=g, device=DEV).double(), _whole(g, (self.room, inter), 2, 0.5)), 1)
        none = torch.ones(self.room, dtype=torch.bool, device=DEV)
        none[before:before + sum(counts)] = False
        for t in (self.x, self.w, self.rows, self.dy, self.kept):
            t[none] = float("nan")

    def forward(self, few):
        """(y, kept), 7 in rows of no expert.  few: h is held as two bf16 values."""
        y, kept = torch.full((self.room, self.hidden), 7.0, device=DEV, dtype=torch.float64), torch.full((self.room, 2, self.inter), 7.0, device=DEV, dtype=torch.float64)
        for e, at in runs(self.counts, self.before):
            x, (gate, up), down = self.x[at], self.gate_up[e], self.down[e]
            g, u = x @ gate.T, x @ up.T
            assert float(g.min()) >= 18
            h = g * u
            _small(h.abs(), "h")
            high = _bf16(h)
            h = high + _bf16(h - high) if few else high
            _small(h.abs() @ down.abs().T, "y")
            y[at], kept[at] = self.w[at, None].double() * (h @ down.T), torch.stack((g, u), 1)
        return y.bfloat16(), kept.bfloat16()

    def backward(self):
        """dx, d_gate_up, d_down, dw; 7 in rows of no expert."""
        dx, dw = torch.full((self.room, self.hidden), 7.0, device=DEV, dtype=torch.float64), torch.full((self.room,), 7.0, device=DEV, dtype=torch.float64)
        d_gate_up, d_down = torch.zeros_like(self.gate_up), torch.zeros_like(self.down)
        for e, at in runs(self.counts, self.before):
            x, dy, w, down, both = self.rows[at], self.dy[at], self.w[at, None].double(), self.down[e], self.gate_up[e].flatten(0, 1)
            g, u = self.kept[at].unbind(1)
            da = dy @ down
            _small(dy.abs() @ down.abs(), "da")
            dw[at] = (da * g * u).sum(1)
            _small((da * g * u).abs().sum(1), "dw")
            h, d = _bf16(w * g * u), _bf16(torch.cat((w * da * u, w * da * g), 1))
            dx[at], d_gate_up[e], d_down[e] = d @ both, (d.T @ x).view(2, self.inter, self.hidden), dy.T @ h
            _small(d.abs() @ both.abs(), "dx"), _small(d.abs().T @ x.abs(), "d_gate_up"), _small(dy.abs().T @ h.abs(), "d_down")
        return dx.bfloat16(), d_gate_up.bfloat16(), d_down.bfloat16(), dw.float()


def codes_of(x):
    """(codes, scales) of rows as the definition has them: 127 x / a to the nearest whole number, halves to even, in 64 bits; a / 127 in single precision (by way of 64 bits: torch divides by a
    number as it multiplies by its reciprocal, which in single precision is another value for six of the 128 significands of a)."""
    a = x.double().abs().amax(1, keepdim=True)
    return torch.where(a > 0, torch.round(127 * x.double() / a), torch.zeros((), dtype=torch.float64, device=x.device)), (a[:, 0] / 127).float()


class CodeBlock:
    """Experts of codes.  Sums of codes are exact in 64 bits; factors come in one after the other in single precision, in the order that the definition names, so results are known to the bit."""

    def __init__(self, counts, hidden, inter, before=0, spare=0, seed=1):
        g = _generator(seed)
        self.counts, self.hidden, self.inter, self.before, self.n = counts, hidden, inter, before, len(counts)
        self.room = before + sum(counts) + spare
        random = lambda most, *shape: torch.randint(-most, most + 1, shape, generator=g, device=DEV, dtype=torch.int8)
        self.gate_up, self.down = random(127, self.n, 2, inter, hidden), random(127, self.n, hidden, inter)
        self.gate_up[:, 0] = random(3, self.n, inter, hidden)
        self.gate_up[:, 0, :, 0] = 100
        self.gate_up_scale, self.down_scale = torch.rand((self.n, 2, inter), generator=g, device=DEV) / 64, torch.rand((self.n, hidden), generator=g, device=DEV)
        self.gate_up_scale[:, 0] = 2.0 ** -8
        self.x, self.w = _whole(g, (self.room, hidden), 4), torch.rand((self.room,), generator=g, device=DEV) - 0.5
        self.x[:, 0] = 127
        self.x *= 2.0 ** torch.randint(0, 3, (self.room, 1), generator=g, device=DEV).double()
        self.x = self.x.bfloat16()
        none = torch.ones(self.room, dtype=torch.bool, device=DEV)
        none[before:before + sum(counts)] = False
        self.x[none], self.w[none] = float("nan"), float("nan")

    def forward(self, weighted=True):
        y = torch.full((self.room, self.hidden), 7.0, device=DEV, dtype=torch.bfloat16)
        for e, at in runs(self.counts, self.before):
            codes, scales = codes_of(self.x[at])
            g, u = ((codes @ self.gate_up[e, k].double().T).float() * scales[:, None] * self.gate_up_scale[e, k] for k in range(2))
            assert float(g.min()) >= 18
            codes, scales = codes_of((g * u).bfloat16())
            v = (codes @ self.down[e].double().T).float() * scales[:, None] * self.down_scale[e]
            y[at] = (self.w[at, None] * v if weighted else v).bfloat16()
        return y


def matrices(counts, n_in, n_out, seed=1, spare=0):
    """codes, scales, w, w_scale, and the product in single precision, 7 in rows of no matrix."""
    g, n, room = _generator(seed), len(counts), sum(counts) + spare
    codes, w = (torch.randint(-127, 128, s, generator=g, device=DEV, dtype=torch.int8) for s in ((room, n_in), (n, n_out, n_in)))
    scales, w_scale = torch.rand((room,), generator=g, device=DEV), torch.rand((n, n_out), generator=g, device=DEV)
    out = torch.full((room, n_out), 7.0, device=DEV)
    for m, at in runs(counts, 0):
        out[at] = (codes[at].double() @ w[m].double().T).float() * scales[at, None] * w_scale[m]
    return codes, scales, w, w_scale, out
