"""mw_moe_layer against a plain 64-bit form.

Tolerances, u = 2^-24: a sum of up to 7168 products is 56 additions of a matrix instruction after another in each of the waves, and
a few more: gamma = 128 u of the sum of sizes.  The activation carries the errors of both products (silu's slope is below 1.1), a few
roundings and its split into two bf16 values (2^-16): 2^-15 of it.  The output is rounded to bf16: 2^-8 of it."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GAMMA = 128 * 2.0 ** -24


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def quantised(w):
    """float32 [..., rows, cols] -> (codes, factors, the values they stand for)."""
    rows, cols = w.shape[-2:]
    f = torch.rand(w.shape[:-2] + (-(-rows // 128), -(-cols // 128)), generator=torch.Generator().manual_seed(9)) * 0.01 + 0.001
    wide = f.repeat_interleave(128, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :cols]
    codes = (w / w.std() * 30).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes, f, codes.double() * wide.double()


class Rank:
    """A rank's experts and context; `fp8`: the weights' format."""

    def __init__(self, n_ranks, E, K, H, I, fp8, my_rank=0, seed=1, max_tokens=256):
        self.e2r = (np.arange(E) % n_ranks).astype(np.int32)             # local experts are not neighbours
        self.slots = {int(e): i for i, e in enumerate(np.nonzero(self.e2r == my_rank)[0])}
        n = len(self.slots)
        up, down = normal(seed, n, 2, I, H) * H ** -0.5, normal(seed + 1, n, H, I) * I ** -0.5
        if fp8:
            (up, us, self.up), (down, ds, self.down) = quantised(up), quantised(down)
            us, ds = us.to(DEV), ds.to(DEV)
        else:
            up, down, us, ds = up.bfloat16(), down.bfloat16(), None, None
            self.up, self.down = up.double(), down.double()
        self.up, self.down = self.up.numpy(), self.down.numpy()
        self.ctx = B.Context(n_ranks, E, K, my_rank, H, B.MW_ROW_BF16, max_tokens, 0, self.e2r)
        self.experts = B.Experts(up.to(DEV), down.to(DEV), us, ds)
        self.E, self.K, self.H = E, K, H

    def run(self, x, ids, w, gate=None, logits=None, bias=None, pad=0, flags=None, out_pad=0):
        T = x.shape[0]
        ws = self.ctx.moe_workspace(self.experts, T)
        ws.fill_(0xff)                                                   # (no part of it has to be prepared)
        out = torch.full((T + 1, self.H + out_pad), 7.0, dtype=torch.bfloat16, device=DEV)
        xd = torch.zeros((T, self.H + pad), dtype=torch.bfloat16, device=DEV)[:, :self.H]
        xd.copy_(x)
        self.ctx.mw_moe_layer(gate, logits, bias, self.experts, xd, ids, w, out[:T, :self.H], ws, flags)
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        assert (got[T] == 7).all() and (got[:, self.H:] == 7).all()
        return got[:T, :self.H]

    def check(self, got, x, ids, w):
        want, off = P.layer(x.double().numpy(), ids, w, self.up, self.down, self.slots, GAMMA)
        bad = ~(np.abs(got - want) <= off + 2.0 ** -8 * np.abs(want) + 1e-30)
        assert not bad.any(), (bad.sum(), np.abs(got - want)[bad].max(), np.argwhere(bad)[:5])


def draw_ids(seed, T, E, K, none=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.rand((T, E), generator=g).topk(K, 1).indices.int()
    ids[torch.rand((T, K), generator=g) < none] = -1
    return ids, torch.rand((T, K), generator=g) + 0.1


SIZES = [(1, 1, 1, 1, 8, 8), (1, 4, 16, 2, 256, 256), (2, 1, 8, 2, 328, 1000), (5, 2, 6, 3, 1000, 136), (13, 2, 16, 2, 512, 264), (16, 1, 4, 4, 128, 128),
         (16, 8, 64, 8, 256, 48), (17, 1, 4, 2, 264, 72), (33, 1, 1, 1, 256, 40), (64, 4, 16, 4, 136, 128), (65, 1, 2, 2, 128, 200), (130, 8, 32, 8, 64, 64),
         (256, 1, 2, 1, 256, 32), (256, 2, 8, 8, 40, 24), (256, 1, 64, 64, 64, 16), (16, 2, 1024, 64, 64, 16)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,R,E,K,H,I", SIZES)
def test_ids_and_weights_given(T, R, E, K, H, I, fp8):
    if fp8:
        H, I = -(-H // 16) * 16, -(-I // 16) * 16
    r = Rank(R, E, K, H, I, fp8)
    x = normal(3, T, H).bfloat16()
    ids, w = draw_ids(T, T, E, K, 0.1)
    got = r.run(x, ids.to(DEV), w.to(DEV), pad=8 * (T % 3), out_pad=8 * (T % 2))
    r.check(got, x, ids.numpy(), w.numpy())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,H,I", [(3, 7168, 144), (20, 272, 2048)])
def test_long_rows(T, H, I, fp8):
    r = Rank(4, 8, 2, H, I, fp8, my_rank=3)
    x = normal(3, T, H).bfloat16()
    ids, w = draw_ids(T, T, 8, 2)
    r.check(r.run(x, ids.to(DEV), w.to(DEV)), x, ids.numpy(), w.numpy())


@pytest.mark.parametrize("T", [1, 7, 16, 40])
def test_from_gate_scores(T):
    r = Rank(4, 32, 4, 256, 128, False)
    gate, x, l = B.Gate(B.MW_GATE_SIGMOID_TOPK, 8, 4, 2.5), normal(5, T, 256).bfloat16(), normal(6, T, 32)
    l[T // 2, 3:] = -float("inf")
    bias = normal(7, 32) * 0.2
    ids, w = torch.full((T, 4), -5, dtype=torch.int32, device=DEV), torch.empty((T, 4), device=DEV)
    got = r.run(x, ids, w, gate, l.to(DEV), bias.to(DEV))
    want_ids, want_w = P.route(l.numpy(), bias.numpy(), 4, P.SIGMOID_TOPK, 8, 4, 2.5)
    np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
    assert (np.abs(w.cpu().numpy() - want_w) <= 64 * 2.0 ** -24 * want_w).all()
    r.check(got, x, want_ids, w.cpu().numpy())


@pytest.mark.parametrize("T", [4, 30])
def test_tokens_that_go_nowhere_here(T):
    """Every expert of a token elsewhere or none: zeros.  No token at all: nothing is written.  A rank without experts: zeros."""
    r = Rank(4, 16, 2, 128, 64, False)
    x = normal(5, T, 128).bfloat16()
    ids, w = torch.full((T, 2), -1, dtype=torch.int32), torch.ones((T, 2))
    ids[1:3] = torch.tensor([1, 2])
    assert (r.run(x, ids.to(DEV), w.to(DEV)) == 0).all()
    ids[3, 1] = 4
    got = r.run(x, ids.to(DEV), w.to(DEV))
    r.check(got, x, ids.numpy(), w.numpy())
    assert (got[:3] == 0).all() and (got[3] != 0).any()
    r.run(x[:0], ids[:0].to(DEV), w[:0].to(DEV))
    idle = Rank(4, 16, 2, 128, 64, False)
    idle.ctx = B.Context(4, 16, 2, 3, 128, B.MW_ROW_BF16, 256, 0, np.zeros(16, dtype=np.int32))
    idle.experts = B.Experts(torch.empty((0, 2, 64, 128), dtype=torch.bfloat16, device=DEV), torch.empty((0, 128, 64), dtype=torch.bfloat16, device=DEV))
    assert (idle.run(x, ids.to(DEV), w.to(DEV)) == 0).all()


@pytest.mark.parametrize("T", [6, 50])
def test_an_expert_named_twice_weighs_both(T):
    r = Rank(1, 4, 3, 136, 72, False)
    x = normal(5, T, 136).bfloat16()
    ids, w = draw_ids(T, T, 4, 3)
    ids[0], ids[1] = torch.tensor([2, 2, 2]), torch.tensor([1, 3, 1])
    r.check(r.run(x, ids.to(DEV), w.to(DEV)), x, ids.numpy(), w.numpy())


@pytest.mark.parametrize("T", [6, 50])
def test_ids_out_of_range_are_left_out_and_flagged(T):
    r = Rank(2, 8, 2, 128, 64, False)
    x = normal(5, T, 128).bfloat16()
    ids, w = draw_ids(T, T, 8, 2)
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    r.check(r.run(x, ids.to(DEV), w.to(DEV), flags=flags), x, ids.numpy(), w.numpy())
    assert int(flags) == 0
    ids[0, 0], ids[1, 1], ids[T - 1, 0], ids[3, 0] = 8, -2, 2 ** 31 - 1, -2 ** 31
    r.check(r.run(x, ids.to(DEV), w.to(DEV), flags=flags), x, ids.numpy(), w.numpy())
    assert int(flags) == B.MW_FLAG_BAD_EXPERT


@pytest.mark.parametrize("T", [9, 40])
def test_values_that_are_no_numbers_stay_where_they_are(T):
    """NaN and infinities in one token and in the weights of one expert reach the tokens they belong to, no other."""
    r = Rank(1, 8, 2, 128, 64, False)
    x = normal(5, T, 128).bfloat16()
    ids, w = draw_ids(T, T, 7, 2)                    # expert 7 unused
    ids[1] = torch.tensor([7, 0])
    r.experts._held[0][7, 0, 3, 5], r.experts._held[1][7, 9] = float("inf"), float("nan")
    x[3, 17] = float("nan")
    x[4, 18] = float("inf")
    w[5, 0] = float("inf")
    got = r.run(x, ids.to(DEV), w.to(DEV))
    assert not np.isfinite(got[1]).all() and not np.isfinite(got[3]).any() and not np.isfinite(got[4]).all() and not np.isfinite(got[5]).any()
    keep = [t for t in range(T) if t not in (1, 3, 4, 5)]
    r.check(got[keep], x[keep], ids.numpy()[keep], w.numpy()[keep])


def test_the_same_calls_give_the_same_bits():
    for T in (16, 100):
        r = Rank(1, 8, 4, 1024, 512, False)
        x, (ids, w) = normal(5, T, 1024).bfloat16(), draw_ids(1, T, 8, 4)
        first = r.run(x, ids.to(DEV), w.to(DEV))
        for _ in range(3):
            np.testing.assert_array_equal(first, r.run(x, ids.to(DEV), w.to(DEV)))


@pytest.mark.parametrize("T", [8, 40])
def test_replayed_from_a_graph_on_another_stream(T):
    r = Rank(2, 16, 2, 256, 128, True)
    gate = B.Gate(B.MW_GATE_SOFTMAX_TOPK)
    x, l = torch.zeros((T, 256), dtype=torch.bfloat16, device=DEV), torch.zeros((T, 16), device=DEV)
    ids, w = torch.empty((T, 2), dtype=torch.int32, device=DEV), torch.empty((T, 2), device=DEV)
    out, ws = torch.empty_like(x), r.ctx.moe_workspace(r.experts, T)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        r.ctx.mw_moe_layer(gate, l, None, r.experts, x, ids, w, out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            r.ctx.mw_moe_layer(gate, l, None, r.experts, x, ids, w, out, ws)
    for seed in range(3):
        xs = normal(20 + seed, T, 256).bfloat16()
        x.copy_(xs)
        l.copy_(normal(30 + seed, T, 16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r.check(out.float().cpu().numpy(), xs, ids.cpu().numpy(), w.cpu().numpy())


def test_refusals():
    r = Rank(2, 8, 2, 128, 64, False, max_tokens=100)
    x, (ids, w) = normal(5, 4, 128).bfloat16().to(DEV), draw_ids(1, 4, 8, 2)
    ids, w, out, ws = ids.to(DEV), w.to(DEV), torch.empty((4, 128), dtype=torch.bfloat16, device=DEV), r.ctx.moe_workspace(r.experts, 4)
    call, good = B._native().mw_moe_layer, [r.ctx._h, 0, None, 0, 0, None, r.experts.address, x, 128, 4, ids, w, out, 128, None, ws, ws.numel(), 0]
    assert call(*good) == B.MW_OK
    wide = torch.zeros(4 * 128 + 8, dtype=torch.bfloat16, device=DEV)
    for at, bad, status in ((1, B.Gate(0).address, B.MW_ERR_INVALID_ARG), (2, x, B.MW_ERR_INVALID_ARG), (6, 0, B.MW_ERR_INVALID_ARG), (7, None, B.MW_ERR_INVALID_ARG),
                            (7, wide[1:], B.MW_ERR_INVALID_ARG), (8, 127, B.MW_ERR_INVALID_ARG), (8, 132, B.MW_ERR_INVALID_ARG), (9, -1, B.MW_ERR_INVALID_ARG),
                            (9, 101, B.MW_ERR_CAPACITY), (10, None, B.MW_ERR_INVALID_ARG), (11, None, B.MW_ERR_INVALID_ARG), (12, None, B.MW_ERR_INVALID_ARG),
                            (12, wide[4:], B.MW_ERR_INVALID_ARG), (13, 120, B.MW_ERR_INVALID_ARG), (15, None, B.MW_ERR_WORKSPACE), (15, ws[16:], B.MW_ERR_WORKSPACE),
                            (16, 255, B.MW_ERR_WORKSPACE), (8, 1 << 29, B.MW_ERR_UNSUPPORTED)):
        assert call(*(good[:at] + [bad] + good[at + 1:])) == status, (at, bad)
    held = r.experts._held
    for change, status in ((dict(inter=0), B.MW_ERR_INVALID_ARG), (dict(inter=60), B.MW_ERR_UNSUPPORTED), (dict(format=2), B.MW_ERR_INVALID_ARG),
                           (dict(format=1), B.MW_ERR_INVALID_ARG), (dict(down_dev=0), B.MW_ERR_INVALID_ARG), (dict(gate_up_dev=held[0].data_ptr() + 8), B.MW_ERR_INVALID_ARG),
                           (dict(down_scale_dev=held[0].data_ptr()), B.MW_ERR_INVALID_ARG)):
        rec = B.MwExperts(*[change.get(f, getattr(r.experts.record, f)) for f, _ in B.MwExperts._fields_])
        assert call(*(good[:6] + [B.C.addressof(rec)] + good[7:])) == status, change
    with pytest.raises(B.MwError) as e:
        r.ctx.moe_workspace(r.experts, 257)
    assert e.value.status == B.MW_ERR_CAPACITY
    for args in ((held[0].float(), held[1]), (held[0][:, :1], held[1]), (held[0], held[1].transpose(1, 2)), (held[0], held[1], torch.ones(1), None)):
        with pytest.raises(ValueError):
            B.Experts(*args)
    with pytest.raises(ValueError):
        r.ctx.mw_moe_layer(None, None, None, r.experts, x.float(), ids, w, out, ws)
    with pytest.raises(ValueError):
        Rank(2, 16, 2, 128, 64, False).ctx.mw_moe_layer(None, None, None, r.experts, x, ids, w, out, ws)
    bytes_ctx = B.Context(2, 8, 2, 0, 128, B.MW_ROW_BYTES, 100, 0, r.e2r, row_bytes=256)
    assert call(*([bytes_ctx._h] + good[1:])) == B.MW_ERR_UNSUPPORTED
    many = B.Context(2, 2048, 2, 0, 128, B.MW_ROW_BF16, 100, 0, np.zeros(2048, dtype=np.int32))
    assert call(*([many._h] + good[1:])) == B.MW_ERR_UNSUPPORTED
