"""mw_quantize_rows and mw_matmul_int8, and mw_ffn with experts of 8-bit codes, against plain 64-bit forms.

Codes are exact.  A product's sum is exact; its conversion to fp32 and the two or three factors are rounded once each: 4 u of the value, u = 2^-24, and 2^-8 for
the rounding to bf16."""
import itertools

import numpy as np
import pytest
import torch

import plain_experts as P
from paper_2605_22428_amd import binding as B
from test_gpu_ffn import DEV, host, near, normal, strided

pytestmark = pytest.mark.gpu


def quantized(x, pad=0):
    codes = torch.full((x.shape[0] + 1, x.shape[1] + pad), 99, dtype=torch.int8, device=DEV)
    scales = torch.full((x.shape[0] + 1,), 7.0, device=DEV)
    B.mw_quantize_rows(x, codes[:-1, :x.shape[1]], scales[:-1])
    torch.cuda.synchronize()
    assert (codes[-1] == 99).all() and (codes[:, x.shape[1]:] == 99).all() and scales[-1] == 7
    return codes[:-1, :x.shape[1]], scales[:-1]


@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 48), (64, 272), (5, 2048), (2, 7168), (3, 8192), (2, 8208), (1, 65536), (1000, 64), (2048, 16), (2051, 2048), (2049, 2064), (2050, 4112), (2048, 8192)])
@pytest.mark.parametrize("pad", [0, 16])
def test_codes(rows, cols, pad):
    x = normal(rows + cols, rows, cols).bfloat16()
    x[0] *= 2.0 ** -100
    codes, scales = quantized(strided(x, pad), pad)
    want, want_scales = P.codes_of(host(x))
    np.testing.assert_array_equal(codes.cpu().numpy(), want)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


def test_codes_of_every_value():
    """All bf16 values up to 1 against the largest values 1, 127 / 128 and 2^-120: halves go to the even code."""
    bits = torch.arange(0x3f81, dtype=torch.int32)
    values = (bits << 16).view(torch.float32)
    for most in (1.0, 127 / 128, 254 / 256, 2.0 ** -120):
        v = values[values <= most]
        v = torch.nn.functional.pad(v, (0, -len(v) % 15))
        x = torch.cat((v.view(15, -1).repeat(2, 1), torch.full((30, 1), most)), 1)
        x[15:] *= -1
        x = torch.nn.functional.pad(x, (0, -x.shape[1] % 16)).bfloat16()
        codes, scales = quantized(x.to(DEV))
        want, want_scales = P.codes_of(host(x))
        np.testing.assert_array_equal(codes.cpu().numpy(), want)
        np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)


def test_rows_of_zeros_and_rows_that_are_not_finite():
    x = normal(1, 6, 32).bfloat16()
    x[1], x[2, 3], x[3, 31], x[4, 0] = 0, float("nan"), float("inf"), -float("inf")
    codes, scales = quantized(x.to(DEV))
    assert (codes[1:5] == 0).all() and scales[1] == 0 and scales[2:5].isnan().all()
    want, want_scales = P.codes_of(host(x))
    for r in (0, 5):
        np.testing.assert_array_equal(codes[r].cpu().numpy(), want[r])
        assert float(scales[r]) == want_scales[r]


class Matrices:
    def __init__(self, n, n_in, n_out, seed=1):
        g = torch.Generator().manual_seed(seed)
        self.w, self.scale = torch.randint(-127, 128, (n, n_out, n_in), generator=g).to(torch.int8), torch.rand((n, n_out), generator=g)
        self.dev = B.MatricesInt8(self.w.to(DEV), self.scale.to(DEV))
        self.n, self.n_in, self.n_out = n, n_in, n_out

    def check(self, counts, spare=0, pad=0, dtype=torch.bfloat16, offsets=True, seed=2):
        g = torch.Generator().manual_seed(seed)
        rows, room = sum(counts), sum(counts) + spare
        codes, scales = torch.randint(-127, 128, (room, self.n_in), generator=g).to(torch.int8), torch.rand((room,), generator=g)
        wide = torch.full((room, self.n_in + 2 * pad), 99, dtype=torch.int8, device=DEV)
        wide[:, :self.n_in] = codes
        out = torch.full((room, self.n_out + pad), 7.0, dtype=dtype, device=DEV)
        at = torch.tensor([0] + list(itertools.accumulate(counts)), device=DEV) if offsets else None
        self.dev.mw_matmul_int8(wide[:, :self.n_in], scales.to(DEV), at, out[:, :self.n_out])
        torch.cuda.synchronize()
        assert (out[rows:] == 7).all() and (out[:, self.n_out:] == 7).all()
        first = 0
        for m, c in enumerate(counts):
            rows_of = slice(first, first + c)
            want = (host(codes[rows_of]) @ host(self.w[m]).T) * host(scales[rows_of])[:, None] * host(self.scale[m])
            near(out[rows_of, :self.n_out], want, 4 * P.U * np.abs(want), P.BF16 if dtype == torch.bfloat16 else 0.0)
            first += c


@pytest.mark.parametrize("counts,n_in,n_out", [([1], 16, 16), ([1], 2048, 272), ([0, 2, 0], 144, 48), ([5, 0, 11], 272, 1008), ([16], 128, 64), ([17, 33], 400, 144), ([64, 65, 63], 256, 128),
                                               ([130], 656, 272), ([256], 128, 256), ([257], 80, 528), ([300, 400], 1040, 304), ([0, 0], 64, 64)])
def test_products(counts, n_in, n_out):
    m = Matrices(len(counts), n_in, n_out)
    m.check(counts, spare=3, pad=16)
    m.check(counts, dtype=torch.float32)
    if len(counts) == 1:
        m.check(counts, offsets=False, dtype=torch.float32, pad=8)


def test_products_of_many_matrices():
    Matrices(100, 64, 48).check([(5 * m) % 4 for m in range(100)], spare=2)
    Matrices(100, 144, 144).check([(7 * m) % 40 if m % 10 == 0 else m % 3 for m in range(100)], spare=2, dtype=torch.float32)


@pytest.mark.parametrize("n,runs", [(40, {3: 600, 39: 33}), (100, {80: 1200, 99: 17, 2: 16}), (70, {0: 33, 64: 1000, 65: 32}), (1, {0: 16}), (700, {5: 70, 250: 17, 699: 1}), (700, {64: 33})])
def test_few_rows_most_of_which_are_one_matrix(n, runs):
    counts = [runs.get(m, 0) for m in range(n)]
    Matrices(n, 144, 80).check(counts, spare=3 if n > 1 else 0, pad=16)


@pytest.mark.parametrize("many", [2, 17 * 66000])
def test_more_matrices_than_a_grid_is_high(many):
    """A few rows of a few of 66000 matrices, and (tiles of many rows) one of them with most."""
    n, counts = 66000, [0] * 66000
    for m in (0, 1, 65534, 65535, 65536, 65999):
        counts[m] = 1 + m % 3
    counts[65700] = many
    s, rows, g = Matrices(n, 16, 16), sum(counts), torch.Generator().manual_seed(4)
    codes = torch.randint(-127, 128, (rows + 3, 16), generator=g).to(torch.int8)
    out = torch.full((rows + 3, 16), 7.0, device=DEV)
    s.dev.mw_matmul_int8(codes.to(DEV), torch.ones(rows + 3, device=DEV), torch.tensor([0] + list(itertools.accumulate(counts)), device=DEV), out)
    torch.cuda.synchronize()
    first = 0
    for m, c in enumerate(counts):
        if c:
            want = host(codes[first:first + c]) @ host(s.w[m]).T * host(s.scale[m])
            near(out[first:first + c], want, 4 * P.U * np.abs(want), 0.0)
            first += c
    assert (out[rows:] == 7).all()


@pytest.mark.parametrize("rows", [1, 20, 130])
def test_a_matrix_larger_than_2_gib(rows):
    """Columns below, around and above the 2 GiB border, whose places in bytes need more than 31 bits."""
    n_in, n_out = 16384, 131072 + 4096
    w = torch.randint(-127, 128, (1, n_out, n_in), dtype=torch.int8, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    scale = torch.rand((1, n_out), device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    codes = torch.randint(-127, 128, (rows, n_in), generator=torch.Generator().manual_seed(3)).to(torch.int8)
    out = torch.full((rows, n_out), 7.0, device=DEV)
    B.MatricesInt8(w, scale).mw_matmul_int8(codes.to(DEV), torch.ones(rows, device=DEV), None, out)
    torch.cuda.synchronize()
    for at in (slice(0, 40), slice(131072 - 300, 131072 + 300), slice(n_out - 40, n_out)):
        want = host(codes) @ host(w[0, at]).T * host(scale[0, at])
        near(out[:, at], want, 4 * P.U * np.abs(want), 0.0)


@pytest.mark.parametrize("rows", [1, 16, 17])
def test_long_rows(rows):
    Matrices(1, 4112, 272).check([rows], spare=1, pad=16)
    Matrices(3, 8208, 48).check([rows, 0, 16], dtype=torch.float32)


@pytest.mark.parametrize("rows", [1, 40, 256])
def test_the_largest_sums(rows):
    """65536 products of -128 and -128 or 127: the largest sums there are, exact in 32 bits."""
    w = torch.full((1, 16, 65536), -128, dtype=torch.int8)
    w[:, 1::2] = 127
    dev = B.MatricesInt8(w.to(DEV), torch.ones((1, 16), device=DEV))
    out = torch.empty((rows, 16), device=DEV)
    dev.mw_matmul_int8(torch.full((rows, 65536), -128, dtype=torch.int8, device=DEV), torch.ones(rows, device=DEV), None, out)
    assert (out[:, ::2] == 2.0 ** 30).all() and (out[:, 1::2] == -128 * 127 * 65536).all()


class Experts:
    def __init__(self, counts, hidden, inter, spare=0, seed=1, weighted=True):
        g, n = torch.Generator().manual_seed(seed), len(counts)
        self.counts, self.hidden, self.inter, self.rows, self.room = counts, hidden, inter, sum(counts), sum(counts) + spare
        self.gate_up, self.down = (torch.randint(-127, 128, s, generator=g).to(torch.int8) for s in ((n, 2, inter, hidden), (n, hidden, inter)))
        self.gate_up_scale, self.down_scale = ((torch.rand(s, generator=g) + 0.5) * k ** -0.5 / 73 for s, k in (((n, 2, inter), hidden), ((n, hidden), inter)))
        self.dev = B.Experts(*(t.to(DEV) for t in (self.gate_up, self.down, self.gate_up_scale, self.down_scale)))
        self.ctx = B.Context(1, n, 1, 0, hidden, B.MW_ROW_BF16, 1, max(self.room, 1), np.zeros(n, dtype=np.int32))
        self.x = normal(seed, self.room, hidden).bfloat16()
        self.x[self.rows:] = float("nan")
        self.w = torch.rand(self.room, generator=g) if weighted else None
        self.offsets = torch.tensor([0] + list(itertools.accumulate(counts)), device=DEV)

    def forward(self, x=None):
        y = torch.full((self.room, self.hidden + 8), 7.0, dtype=torch.bfloat16, device=DEV)
        ws = self.ctx.ffn_workspace(self.dev, self.room)
        ws.fill_(0xff)
        self.ctx.mw_ffn(self.dev, strided(self.x, 8) if x is None else x, self.offsets, y[:, :self.hidden], ws, None if self.w is None else self.w.to(DEV))
        torch.cuda.synchronize()
        assert (y[self.rows:] == 7).all() and (y[:, self.hidden:] == 7).all()
        return y[:self.rows, :self.hidden]

    def check(self):
        """h is rounded to bf16, then to codes: where its exact value is within fp32 roundings (32 u) of the middle of two bf16 values it may be either, and a code made of it
        another one; both roundings' ends bound the sum."""
        y, first = self.forward(), 0
        for e, c in enumerate(self.counts):
            at = slice(first, first + c)
            first += c
            if not c:
                continue
            codes, scales = P.codes_of(host(self.x[at]))
            gu = host(self.gate_up[e]) * 1.0
            g, u = ((codes @ gu[k].T) * scales.astype(np.float64)[:, None] * host(self.gate_up_scale[e, k]) for k in range(2))
            h = g * P.sig(g) * u
            low, high = P.bf16(h - 32 * P.U * np.abs(h)), P.bf16(h + 32 * P.U * np.abs(h))
            middle = P.bf16(h)
            q, s = P.codes_of(middle)
            a = np.abs(middle).max(1, keepdims=True)
            # a row whose largest value may round either way may have another scale
            a_off = np.maximum(np.abs(np.abs(low).max(1, keepdims=True) - a), np.abs(np.abs(high).max(1, keepdims=True) - a))
            loose = (np.maximum(np.abs(low - middle), np.abs(high - middle)) > 0) | (a_off > 0)
            # the value that a loose code stands for is off by at most a step, its own change and the change of the step
            off_h = loose * (a / 127 + np.abs(high - low) + a_off)
            w = np.ones(c) if self.w is None else host(self.w[at])
            down = host(self.down[e]) * host(self.down_scale[e])[:, None]
            # (products of codes and their sums are whole numbers, exact here: factors inside the sum would leave 2^-53 of its terms where they cancel)
            want = w[:, None] * (q @ host(self.down[e]).T) * s.astype(np.float64)[:, None] * host(self.down_scale[e])
            near(y[at], want, np.abs(w)[:, None] * (off_h @ np.abs(down).T) + 6 * P.U * np.abs(want))


@pytest.mark.parametrize("counts,hidden,inter", [([1], 16, 16), ([2, 0, 1], 256, 144), ([9, 5], 1040, 272), ([40, 0, 70], 272, 400), ([300], 400, 144), ([257, 400], 144, 256), ([300, 0, 290], 2064, 1040), ([3, 60], 2064, 2080)])
def test_experts(counts, hidden, inter):
    Experts(counts, hidden, inter, spare=3).check()
    Experts(counts, hidden, inter, weighted=False, seed=5).check()


def test_a_row_that_is_not_finite_stays_by_itself():
    for counts in ([3, 4], [60, 70], [250, 260]):
        s = Experts(counts, 144, 80)
        want = s.forward()
        x = s.x.to(DEV)
        x[2, 7] = float("inf")
        got = s.forward(x)
        others = [r for r in range(s.rows) if r != 2]
        assert torch.equal(got[others], want[others]) and got[2].isnan().all()


@pytest.mark.parametrize("counts", [[2, 1], [40, 50], [300, 400]])
def test_replayed_from_a_graph_on_another_stream(counts):
    s = Experts(counts, 144, 80, spare=2)
    m = Matrices(2, 144, 64)
    x, w, y, ws = torch.zeros((s.room, 144), dtype=torch.bfloat16, device=DEV), s.w.to(DEV), torch.empty((s.room, 144), dtype=torch.bfloat16, device=DEV), s.ctx.ffn_workspace(s.dev, s.room)
    codes, scales, out = torch.empty((s.room, 144), dtype=torch.int8, device=DEV), torch.empty(s.room, device=DEV), torch.empty((s.room, 64), device=DEV)
    st = torch.cuda.Stream()

    def step():
        s.ctx.mw_ffn(s.dev, x, s.offsets, y, ws, w)
        B.mw_quantize_rows(y, codes, scales)
        m.dev.mw_matmul_int8(codes, scales, s.offsets, out)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
    for seed in range(4):
        x.copy_(normal(60 + seed, s.room, 144).bfloat16())
        s.offsets.copy_(torch.tensor([0, counts[0] - seed % 2, s.rows]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t[:s.rows].clone() for t in (y, codes, scales, out)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b[:s.rows]) for a, b in zip(got, (y, codes, scales, out)))
        assert torch.equal(got[0], s.forward(x)) or s.w is None


def test_refusals_of_experts():
    s = Experts([2], 64, 32)
    y, kept, ws = torch.empty((2, 64), dtype=torch.bfloat16, device=DEV), torch.empty((2, 2, 32), dtype=torch.bfloat16, device=DEV), s.ctx.ffn_workspace(s.dev, 2)
    x = s.x.to(DEV)
    for call, status in ((lambda: s.ctx.mw_ffn(s.dev, x, s.offsets, y, ws, None, kept), B.MW_ERR_INVALID_ARG), (lambda: s.ctx.ffn_workspace(s.dev, 2, True), B.MW_ERR_UNSUPPORTED),
                         (lambda: s.ctx.mw_ffn_backward(s.dev, x, s.offsets, kept, x, y, None, None, ws), B.MW_ERR_UNSUPPORTED)):
        with pytest.raises(B.MwError) as e:
            call()
        assert e.value.status == status
    for change, status in ((dict(inter=24), B.MW_ERR_UNSUPPORTED), (dict(gate_up_scale_dev=0), B.MW_ERR_INVALID_ARG), (dict(down_scale_dev=s.dev.record.down_scale_dev + 2), B.MW_ERR_INVALID_ARG)):
        rec = B.MwExperts(*[change.get(f, getattr(s.dev.record, f)) for f, _ in B.MwExperts._fields_])
        assert B._native().mw_ffn(s.ctx._h, B.C.addressof(rec), x, 64, s.offsets, 2, None, y, 64, None, ws, ws.numel(), 0) == status, change
    c = B.Context(1, 1, 1, 0, 64, B.MW_ROW_BF16, 4, 4, np.zeros(1, dtype=np.int32))
    with pytest.raises(B.MwError) as e:
        c.moe_workspace(s.dev, 4)
    assert e.value.status == B.MW_ERR_INVALID_ARG
