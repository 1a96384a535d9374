"""mw_adapt and mw_adapt_backward against a plain 64-bit form.

Tolerances, u = 2^-24: a sum of products is at most 7168 / 32 / 8 additions of a matrix instruction in a wave, or 256 of rows, and a few
more: gamma = 300 u of the sum of sizes.  What goes from the first product into the second is split into two bf16 values (2^-16, with the
factor's rounding 2^-15).  bf16 results are rounded once more: 2^-8 of the value."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GAMMA = 300 * 2.0 ** -24


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


class Set:
    def __init__(self, n, rank, n_in, n_out, scaled=True, seed=1):
        a, b = (normal(seed, n, rank, n_in) * n_in ** -0.5).bfloat16(), (normal(seed + 1, n, n_out, rank) * rank ** -0.5).bfloat16()
        scale = torch.rand((n,), generator=torch.Generator().manual_seed(seed)) + 0.5 if scaled else None
        self.a, self.b = a.double().numpy(), b.double().numpy()
        self.scale = scale.double().numpy() if scaled else np.ones(n)
        self.dev = B.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV) if scaled else None)
        self.n, self.rank, self.n_in, self.n_out = n, rank, n_in, n_out

    def forward(self, x, ids, base, pad=0, in_place=False, keep_h=True, flags=None):
        T = len(ids)
        out = torch.full((T + 1, self.n_out + pad), 7.0, dtype=torch.bfloat16, device=DEV)
        h = torch.full((T + 1, self.rank), 7.0, device=DEV) if keep_h else None
        ws = self.dev.workspace(T, False)
        ws.fill_(0xff)                                                   # (no part of it has to be prepared)
        y = out[:T, :self.n_out]
        base_dev = None if base is None else strided(base, 2 * pad)
        if in_place:
            y.copy_(base_dev)
            base_dev = y
        self.dev.mw_adapt(strided(x, pad), torch.from_numpy(ids).to(DEV), base_dev, y, ws, None if h is None else h[:T], flags)
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        assert (got[T] == 7).all() and (got[:, self.n_out:] == 7).all() and (h is None or (h[T] == 7).all())
        return got[:T, :self.n_out], None if h is None else h[:T].cpu().numpy()

    def check(self, x, ids, base, **kw):
        got, h = self.forward(x, ids, base, **kw)
        base64 = np.zeros((len(ids), self.n_out)) if base is None else base.double().numpy()
        want, want_h, off, off_h = P.adapt(x.double().numpy(), ids, base64, self.a, self.b, self.scale, GAMMA)
        close(got, want, off)
        if h is not None:
            assert (np.abs(h - want_h) <= off_h + 1e-30).all()


def close(got, want, off):
    bad = ~(np.abs(got - want) <= off + 2.0 ** -8 * np.abs(want) + 1e-30)
    assert not bad.any(), (bad.sum(), np.abs(got - want)[bad].max(), np.argwhere(bad)[:5])


def mixed(seed, T, n, none=0.2):
    g = np.random.default_rng(seed)
    ids = g.integers(0, n, T).astype(np.int32)
    ids[g.random(T) < none] = -1
    return ids


SIZES = [(1, 1, 8, 8, 8), (1, 3, 16, 256, 264), (2, 5, 8, 136, 1000), (7, 2, 24, 328, 72), (31, 1, 32, 128, 128), (33, 1, 40, 264, 328), (64, 24, 16, 512, 256),
         (65, 64, 64, 72, 88), (130, 3, 96, 256, 64), (200, 2, 128, 136, 200), (257, 7, 16, 40, 24), (600, 300, 8, 64, 16), (1500, 1024, 8, 16, 16)]


@pytest.mark.parametrize("T,n,rank,n_in,n_out", SIZES)
def test_forward(T, n, rank, n_in, n_out):
    s = Set(n, rank, n_in, n_out, scaled=T % 2 == 0)
    x, base = normal(5, T, n_in).bfloat16(), normal(6, T, n_out).bfloat16()
    ids = mixed(T, T, n)
    s.check(x, ids, base, pad=8 * (T % 3))
    s.check(x, np.sort(ids), None, keep_h=False)
    s.check(x, ids, base, pad=16, in_place=True)


@pytest.mark.parametrize("T,n,rank,n_in,n_out", [(3, 2, 16, 7168, 256), (40, 2, 64, 4096, 1024), (5, 2, 8, 264, 7168)])
def test_long_rows(T, n, rank, n_in, n_out):
    s = Set(n, rank, n_in, n_out)
    s.check(normal(5, T, n_in).bfloat16(), mixed(T, T, n), normal(6, T, n_out).bfloat16())


@pytest.mark.parametrize("T", [5, 64, 300, 5000])
def test_rows_of_one_adapter_or_none(T):
    s = Set(3, 16, 64, 48)
    x, base = normal(5, T, 64).bfloat16(), normal(6, T, 48).bfloat16()
    got, h = s.forward(x, np.full(T, -1, dtype=np.int32), base)
    assert (got == base.float().numpy()).all() and (h == 0).all()
    got, _ = s.forward(x, np.full(T, -1, dtype=np.int32), None)
    assert (got == 0).all()
    s.check(x, np.full(T, 2, dtype=np.int32), base)
    s.check(x, (np.arange(T) % 3).astype(np.int32), base)


def test_many_rows():
    """Rows in order, in no order, and as many as a call takes."""
    s = Set(5, 8, 16, 16)
    for T in (8192, 65536):
        ids = mixed(T, T, 5)
        s.check(normal(5, T, 16).bfloat16(), ids, normal(6, T, 16).bfloat16())


@pytest.mark.parametrize("T", [6, 100])
def test_ids_out_of_range_have_no_adapter_and_are_flagged(T):
    s = Set(4, 16, 64, 64)
    x, base, ids = normal(5, T, 64).bfloat16(), normal(6, T, 64).bfloat16(), mixed(T, T, 4)
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    s.check(x, ids, base, flags=flags)
    assert int(flags) == 0
    ids[[0, 2, T - 1]] = 4, -2, 2 ** 31 - 1
    s.check(x, ids, base, flags=flags)
    assert int(flags) == B.MW_FLAG_BAD_ADAPTER


def test_values_that_are_no_numbers_stay_in_their_row():
    s = Set(3, 16, 64, 64)
    T = 40
    x, base, ids = normal(5, T, 64).bfloat16(), normal(6, T, 64).bfloat16(), mixed(1, T, 2, 0.0)
    x[4, 3], x[5, 6], base[6, 1] = float("nan"), float("inf"), float("inf")
    ids[7], ids[8] = 2, -1
    x[8] = float("nan")                                                 # a row without an adapter: its input does not matter
    s.dev._held[0][2, 1, 1] = float("nan")
    got, h = s.forward(x, ids, base)
    assert not np.isfinite(got[4]).any() and not np.isfinite(got[5]).any() and np.isinf(got[6, 1]) and not np.isfinite(got[7]).any()
    keep = [t for t in range(T) if t not in (4, 5, 6, 7, 8)]
    want, _, off, _ = P.adapt(x.double().numpy()[keep], ids[keep], base.double().numpy()[keep], s.a, s.b, s.scale, GAMMA)
    close(got[keep], want, off)
    assert (got[8] == base[8].float().numpy()).all() and (h[8] == 0).all()


def backward(s, x, ids, h, dy, dx_base, pad=0, in_place=False):
    T = len(ids)
    dx = torch.full((T + 1, s.n_in + pad), 7.0, dtype=torch.bfloat16, device=DEV)
    da, db = torch.full((s.n, s.rank, s.n_in), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((s.n, s.n_out, s.rank), 7.0, dtype=torch.bfloat16, device=DEV)
    base = None if dx_base is None else strided(dx_base, pad)
    to = dx[:T, :s.n_in]
    if in_place:
        to.copy_(base)
        base = to
    ws = s.dev.workspace(T)
    ws.fill_(0xff)
    s.dev.mw_adapt_backward(strided(x, pad), torch.from_numpy(ids).to(DEV), torch.from_numpy(h).to(DEV), strided(dy, 2 * pad), base, to, da, db, ws)
    torch.cuda.synchronize()
    got = dx.float().cpu().numpy()
    assert (got[T] == 7).all() and (got[:, s.n_in:] == 7).all()
    return got[:T, :s.n_in], da.float().cpu().numpy(), db.float().cpu().numpy()


@pytest.mark.parametrize("T,n,rank,n_in,n_out", SIZES[:12])
def test_gradients_against_the_formulas(T, n, rank, n_in, n_out):
    s = Set(n, rank, n_in, n_out, scaled=T % 2 == 1)
    x, dy, dxb, ids = normal(5, T, n_in).bfloat16(), normal(6, T, n_out).bfloat16(), normal(7, T, n_in).bfloat16(), mixed(T, T, n)
    h = (normal(8, T, rank) * (torch.from_numpy(ids) >= 0)[:, None]).numpy()
    for base, kw in ((dxb, dict(pad=8 * (T % 3))), (None, {}), (dxb, dict(pad=8, in_place=True))):
        got = backward(s, x, ids, h, dy, base, **kw)
        base64 = np.zeros((T, n_in)) if base is None else base.double().numpy()
        want = P.adapt_backward(x.double().numpy(), ids, h.astype(np.float64), dy.double().numpy(), base64, s.a, s.b, s.scale, GAMMA)
        for g, (w, off) in zip(got, want):
            close(g, w, off)
    for a in set(range(n)) - set(ids.tolist()):
        assert (got[1][a] == 0).all() and (got[2][a] == 0).all()


@pytest.mark.parametrize("T,n,rank,n_in,n_out", [(3000, 2, 64, 136, 264), (5, 2, 16, 7168, 4096), (700, 1, 128, 256, 512), (70, 1024, 8, 24, 16)])
def test_gradients_of_many_rows_and_long_rows(T, n, rank, n_in, n_out):
    s = Set(n, rank, n_in, n_out)
    x, dy, ids, h = normal(5, T, n_in).bfloat16(), normal(6, T, n_out).bfloat16(), mixed(T, T, n, 0.1), normal(8, T, rank).numpy()
    got = backward(s, x, ids, h, dy, None)
    want = P.adapt_backward(x.double().numpy(), ids, h.astype(np.float64), dy.double().numpy(), np.zeros((T, n_in)), s.a, s.b, s.scale, GAMMA)
    for g, (w, off) in zip(got, want):
        close(g, w, off)


def test_gradients_of_no_rows_are_zero():
    s = Set(2, 8, 16, 24)
    none = np.zeros(0, dtype=np.int32)
    _, da, db = backward(s, torch.empty((0, 16), dtype=torch.bfloat16), none, np.zeros((0, 8), dtype=np.float32), torch.empty((0, 24), dtype=torch.bfloat16), None)
    assert (da == 0).all() and (db == 0).all()


def test_gradients_against_differences():
    """L = sum of g out; central differences of the kernel's own forward in the direction of a perturbation v of x, A and B.  L is a polynomial
    of degree 3 in the step along v, so a central difference with step e is off by e^2 times its cubic term; out is rounded to bf16 (2^-9
    of its size each, at random signs: their sum over N outputs stays below 6 sqrt(N) times that)."""
    T, n, rank, n_in, n_out, step = 48, 3, 8, 64, 32, 2.0 ** -3
    s = Set(n, rank, n_in, n_out)
    x, g, ids = normal(5, T, n_in).bfloat16(), normal(6, T, n_out).bfloat16(), mixed(3, T, n, 0.1)
    _, h = s.forward(x, ids, None)
    dx, da, db = backward(s, x, ids, h, g, None)
    a, b = s.dev._held[0].cpu(), s.dev._held[1].cpu()
    for k, (value, grad) in enumerate(((x, dx), (a, da), (b, db))):
        v = (torch.randint(0, 2, value.shape, generator=torch.Generator().manual_seed(k)) * 2 - 1).float() * value.float().abs()
        ends, noise, moved = [], 0.0, []
        for sign in (1, -1):
            at = (value.float() + sign * step * v).bfloat16()
            moved.append(at.double())
            parts = [x, a, b]
            parts[k] = at
            t = Set.__new__(Set)
            t.__dict__.update(s.__dict__)
            t.dev = B.Adapters(parts[1].to(DEV), parts[2].to(DEV), s.dev._held[2])
            out, _ = t.forward(parts[0], ids, None)
            ends.append((out.astype(np.float64) * g.double().numpy()).sum())
            noise += ((np.abs(out) * np.abs(g.float().numpy())) ** 2).sum()
        # L is linear in each of the three alone: the difference along the step as it was rounded is the gradient's product with it
        along = (moved[0] - moved[1]).numpy()
        want = (grad.astype(np.float64) * along).sum()
        slack = 6 * 2.0 ** -9 * (np.sqrt(noise) + np.sqrt(((grad * along) ** 2).sum()))
        assert abs((ends[0] - ends[1]) - want) <= slack, (k, ends, want, slack)


def test_equal_calls_give_equal_bits():
    s = Set(3, 32, 512, 256)
    T = 900
    x, dy, ids, h = normal(5, T, 512).bfloat16(), normal(6, T, 256).bfloat16(), mixed(T, T, 3), normal(8, T, 32).numpy()
    first = backward(s, x, ids, h, dy, None) + s.forward(x, ids, None)
    for _ in range(3):
        for u, v in zip(first, backward(s, x, ids, h, dy, None) + s.forward(x, ids, None)):
            np.testing.assert_array_equal(u, v)


@pytest.mark.parametrize("T", [8, 300])
def test_replayed_from_a_graph_on_another_stream(T):
    s = Set(4, 16, 256, 128)
    x, base, dy = (torch.zeros((T, w), dtype=torch.bfloat16, device=DEV) for w in (256, 128, 128))
    ids, out, h = torch.zeros(T, dtype=torch.int32, device=DEV), torch.empty_like(base), torch.empty((T, 16), device=DEV)
    dx, da, db, ws = torch.empty_like(x), torch.empty_like(s.dev._held[0]), torch.empty_like(s.dev._held[1]), s.dev.workspace(T)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        s.dev.mw_adapt(x, ids, base, out, ws, h)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            s.dev.mw_adapt(x, ids, base, out, ws, h)
            s.dev.mw_adapt_backward(x, ids, h, dy, None, dx, da, db, ws)
    for seed in range(3):
        xs, bs, ds, i = normal(20 + seed, T, 256).bfloat16(), normal(30 + seed, T, 128).bfloat16(), normal(40 + seed, T, 128).bfloat16(), mixed(seed, T, 4)
        for to, v in ((x, xs), (base, bs), (dy, ds), (ids, torch.from_numpy(i))):
            to.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, _, off, _ = P.adapt(xs.double().numpy(), i, bs.double().numpy(), s.a, s.b, s.scale, GAMMA)
        close(out.float().cpu().numpy(), want, off)
        want = P.adapt_backward(xs.double().numpy(), i, h.double().cpu().numpy(), ds.double().numpy(), np.zeros((T, 256)), s.a, s.b, s.scale, GAMMA)
        for g, (w, off) in zip((dx, da, db), want):
            close(g.float().cpu().numpy(), w, off)


def test_refusals():
    s, T = Set(2, 16, 64, 32), 4
    x, ids, out, h = normal(1, T, 64).bfloat16().to(DEV), torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros((T, 32), dtype=torch.bfloat16, device=DEV), torch.zeros((T, 16), device=DEV)
    ws, wide = s.dev.workspace(T), torch.zeros(4096, dtype=torch.bfloat16, device=DEV)
    da, db = torch.empty_like(s.dev._held[0]), torch.empty_like(s.dev._held[1])
    I, CAP, WS, UN = B.MW_ERR_INVALID_ARG, B.MW_ERR_CAPACITY, B.MW_ERR_WORKSPACE, B.MW_ERR_UNSUPPORTED
    call, good = B._native().mw_adapt, [s.dev.address, x, 64, ids, T, None, 0, out, 32, None, None, ws, ws.numel(), 0]
    assert call(*good) == B.MW_OK
    for at, bad, status in ((2, 1 << 29, UN), (8, 1 << 29, UN), (0, 0, I), (1, None, I), (1, wide[4:], I), (2, 56, I), (2, 68, I), (3, None, I), (4, -1, I), (4, 65537, CAP), (5, wide[1:], I), (5, out, I),
                            (7, None, I), (8, 24, I), (11, None, WS), (11, ws[8:], WS), (12, 100, WS)):
        assert call(*(good[:at] + [bad] + good[at + 1:])) == status, (at, bad)
    back, good_b = B._native().mw_adapt_backward, [s.dev.address, x, 64, ids, T, h, out, 32, None, 0, x, 64, da, db, None, ws, ws.numel(), 0]
    for at, bad, status in ((2, 1 << 29, UN), (7, 1 << 29, UN), (11, 1 << 29, UN), (0, 0, I), (1, None, I), (2, 56, I), (3, None, I), (4, -1, I), (4, 65537, CAP), (5, None, I), (6, None, I), (7, 28, I), (8, x, I), (10, None, I),
                            (11, 0, I), (12, None, I), (13, None, I), (13, wide[1:], I), (15, None, WS), (16, 0, WS)):
        assert back(*(good_b[:at] + [bad] + good_b[at + 1:])) == status, (at, bad)
    for change, status in ((dict(rank=12), UN), (dict(rank=136), UN), (dict(rank=0), I), (dict(n_in=60), UN), (dict(n_out=36), UN), (dict(n_adapters=0), I),
                           (dict(n_adapters=1025), UN), (dict(a_dev=0), I), (dict(b_dev=s.dev.record.b_dev + 2), I), (dict(n_in=-8), I)):
        rec = B.MwAdapters(*[change.get(f, getattr(s.dev.record, f)) for f, _ in B.MwAdapters._fields_])
        assert call(*([B.C.addressof(rec)] + good[1:])) == status, change
    with pytest.raises(B.MwError) as e:
        s.dev.workspace(65537)
    assert e.value.status == CAP
    for args in ((x.float(), ids, None, out, ws), (x, ids.long(), None, out, ws), (x, ids[:3], None, out, ws), (x, ids, out[:, :8], out, ws), (x[:, ::2], ids, None, out, ws),
                 (x, ids, None, out[:3], ws), (x, ids, None, out, ws, h[:, :8])):
        with pytest.raises(ValueError):
            s.dev.mw_adapt(*args)
    with pytest.raises(ValueError):
        B.Adapters(da.float(), db)
    with pytest.raises(ValueError):
        B.Adapters(da, db[:1])
