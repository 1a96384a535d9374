"""mw_route and mw_route_backward against a plain 64-bit form: ids exactly, weights and gradients within rounding.

Tolerances, u = 2^-24: a weight is exp(l - m) (the difference is off by u |l - m| <= 30 u here, the function by 2 u), a sum of at
most 16 + 6 partial sums (22 u), a division and a product: 64 u covers it.  A gradient adds one more such weight and a
difference: 128 u of the sizes of what is added up.  bf16 gradients are rounded once more: 2^-8 of the value."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TINY = 2.0 ** -126


def make_ctx(E, K, max_tokens=64):
    return B.Context(1, E, K, 0, 8, B.MW_ROW_BF16, max_tokens, 0, np.zeros(E, dtype=np.int32))


def scores(T, E, seed, dtype, pad=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn((T, E + pad), generator=g).to(dtype).to(DEV)
    return t[:, :E]


def run_route(ctx, gate, logits, bias):
    n = logits.shape[0]
    ids = torch.full((n + 1, ctx.top_k), -77, dtype=torch.int32, device=DEV)
    w = torch.full((n + 1, ctx.top_k), -77.0, device=DEV)
    ctx.mw_route(gate, logits, bias, ids[:n], w[:n])
    torch.cuda.synchronize()
    assert (ids[n] == -77).all() and (w[n] == -77).all()
    return ids[:n].cpu().numpy(), w[:n].cpu().numpy()


def check_route(logits, bias, K, score, groups=1, kept=1, scale=1.0, max_tokens=64):
    ctx = make_ctx(logits.shape[1], K, max(max_tokens, logits.shape[0]))
    ids, w = run_route(ctx, B.Gate(score, groups, kept, scale), logits, bias)
    want_ids, want = P.route(logits.float().cpu().numpy(), None if bias is None else bias.cpu().numpy(), K, score, groups, kept, scale)
    np.testing.assert_array_equal(ids, want_ids)
    assert (np.abs(w - want) <= 64 * U * np.abs(want) + TINY).all(), np.abs(w / np.where(want, want, 1) - 1).max()
    ctx.close()


SHAPES = [(1, 1, 1, 1, 1), (1, 8, 2, 1, 1), (5, 16, 2, 4, 2), (7, 60, 4, 1, 1), (64, 64, 8, 8, 4), (3, 64, 64, 1, 1), (9, 65, 5, 1, 1), (9, 160, 6, 8, 3),
          (33, 256, 8, 8, 4), (10, 256, 8, 64, 8), (4, 384, 9, 1, 1), (6, 1000, 20, 1, 1), (5, 1024, 64, 2, 1), (3, 1024, 8, 64, 1), (4, 6, 3, 6, 4),
          (301, 128, 6, 1, 1)]


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
@pytest.mark.parametrize("T,E,K,G,kept", SHAPES)
def test_ids_and_weights(T, E, K, G, kept, score):
    for dtype, bias, pad in ((torch.float32, False, 0), (torch.float32, True, 3), (torch.bfloat16, True, 1)):
        l = scores(T, E, T + E + score, dtype, pad)
        b = scores(1, E, 5, torch.float32)[0].contiguous() * 0.3 if bias else None
        check_route(l, b, K, score, G, kept, 2.5)


@pytest.mark.parametrize("G,kept", [(1, 1), (8, 3)])
def test_equal_scores_go_to_the_lowest(G, kept):
    """Scores of five values, of both zeros among them: nearly every choice is among equals."""
    g = torch.Generator().manual_seed(3)
    l = torch.randint(-2, 3, (40, 256), generator=g).float() * torch.tensor(1.0)
    l[::2] *= -1.0                                  # (-0 too)
    check_route(l.to(DEV), None, 12, P.SOFTMAX_TOPK, G, kept)
    check_route(torch.zeros((3, 256), device=DEV), None, 12, P.SIGMOID_TOPK, G, kept)


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
@pytest.mark.parametrize("G,kept", [(1, 1), (4, 2)])
def test_masked_experts_and_values_that_are_no_numbers(score, G, kept):
    inf, nan, low = float("inf"), float("nan"), float(torch.finfo(torch.float32).min)
    l = scores(14, 64, 1, torch.float32).clone()
    l[0] = -inf                                     # nothing left
    l[1] = nan
    l[2, 3:] = -inf                                 # fewer than top_k
    l[3, ::2] = -inf
    l[4, 7] = nan
    l[5, 9] = inf
    l[6, 9], l[6, 40] = inf, inf
    l[7] = low                                      # masked by the lowest value
    l[8, 1:] = low
    l[9, :32] = low
    l[10] = low
    l[10, 5] = -inf
    l[11, 16:] = -inf                               # one group
    l[12, ::16] = inf
    l[13, 20] = low
    check_route(l, None, 8, score, G, kept)
    b = torch.zeros(64, device=DEV)
    b[10:20], b[30], b[31], b[32] = -inf, nan, low, inf
    check_route(l, b, 8, score, G, kept)


def test_batches_of_every_size_leave_other_rows_alone():
    for T in (1, 3, 4, 5, 64):
        check_route(scores(T, 32, T, torch.float32), None, 4, P.SOFTMAX)


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
@pytest.mark.parametrize("T,E,K", [(1, 1, 1), (3, 8, 2), (9, 60, 4), (5, 64, 64), (33, 256, 8), (4, 1000, 20), (2, 1024, 8)])
def test_gradient_against_the_formula(T, E, K, score):
    for dtype in (torch.float32, torch.bfloat16):
        ctx = make_ctx(E, K)
        l = scores(T, E, 11 + T, dtype, 2)
        if E > 4:
            l[0, 3] = -float("inf")
            l[T // 2, E // 2] = float("nan")
        gate = B.Gate(score, 1, 1, 1.5)
        ids, _ = run_route(ctx, gate, l, None)
        dw = scores(T, K, 12, torch.float32).contiguous()
        if K > 2:
            ids[0, 1] = -1                          # a token that lost an expert (its gradient is not a number)
            dw[0, 1] = float("nan")
            ids[T - 1, 2] = E
        out = torch.full((T + 1, E + 2), -9.0, dtype=dtype, device=DEV)
        ctx.mw_route_backward(gate, l, torch.from_numpy(ids).to(DEV), dw, out[:T, :E])
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        assert (got[T] == -9).all() and (got[:, E:] == -9).all()
        want, size = P.route_backward(l.float().cpu().numpy(), ids, np.nan_to_num(dw.cpu().numpy()), score, 1.5)
        tol = 128 * U * size + TINY + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0)
        assert (np.abs(got[:T, :E] - want) <= tol).all()
        ctx.close()


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
def test_gradient_against_differences(score):
    """Central differences of mw_route's weights with a step of 2^-5.  Third derivatives of these weights are below 2 c: the formula's
    error is below 2 c step^2 / 6 a weight; rounding adds 64 u c / step."""
    T, E, K, step, c = 4, 24, 5, 2.0 ** -5, 1.5
    ctx, gate = make_ctx(E, K, 2 * E * T), B.Gate(score, 1, 1, c)
    l = scores(T, E, 2, torch.float32).contiguous()
    l += torch.arange(E, device=DEV).flip(0) * 0.5     # (the choice stays the same under the step)
    ids, _ = run_route(ctx, gate, l, None)
    dw = scores(T, K, 8, torch.float32).contiguous()
    out = torch.empty_like(l)
    ctx.mw_route_backward(gate, l, torch.from_numpy(ids).to(DEV), dw, out)
    eye = torch.eye(E, device=DEV) * step
    both = torch.cat([l[:, None] + eye, l[:, None] - eye]).view(-1, E).contiguous()
    at, w = run_route(ctx, gate, both, None)
    by_id = np.zeros((len(at), E + 1))
    np.put_along_axis(by_id, at.astype(np.int64), w.astype(np.float64), 1)
    v = by_id.reshape(2, T, E, E + 1)
    g = np.zeros((T, E + 1))
    np.put_along_axis(g, ids.astype(np.int64), dw.cpu().numpy().astype(np.float64), 1)
    stays = (np.sort(at.reshape(2, T, E, K), -1) == np.sort(ids, -1)[None, :, None]).all(-1).all(0)
    assert stays.mean() > 0.7
    want = ((v[0] - v[1]) / (2 * step) * g[:, None]).sum(-1)
    tol = (2 * c * step ** 2 / 6 + 64 * U * c / step) * np.abs(g).sum(1)[:, None]
    assert (np.abs(out.cpu().numpy() - want) <= tol)[stays].all()
    ctx.close()


def test_ids_feed_the_plan():
    """Scores -> ids -> destination bitmaps: the plan of the ids mw_route writes is the plan of the plain form's ids."""
    from oracle import ref
    import gpu_harness as H
    e2r = (np.arange(64) // 8).astype(np.int32)
    ctx = B.Context(8, 64, 6, 0, 64, B.MW_ROW_BF16, 100, 0, e2r)
    l = scores(100, 64, 4, torch.float32)
    l[50] = -float("inf")
    ids = torch.empty((100, 6), dtype=torch.int32, device=DEV)
    w = torch.empty((100, 6), device=DEV)
    buf = B.SendBuffers(ctx, 100)
    ctx.mw_route(B.Gate(B.MW_GATE_SIGMOID_TOPK, 8, 3), l, None, ids, w)
    ctx.mw_plan(ids, buf.mask, buf.perm, buf.desc, buf.stats)
    want, _ = P.route(l.cpu().numpy(), None, 6, P.SIGMOID_TOPK, 8, 3)
    mask, perm, desc, _ = ref.plan(want, e2r, 8, 128)
    H.assert_same_bytes(H.host(buf.mask).view(np.uint64)[:100], mask, "mask")
    assert int(ctx.mw_get_send_stats(buf.stats)["n_rows"]) == len(perm) == 99


def test_replayed_from_a_graph_on_another_stream():
    ctx, gate = make_ctx(256, 8), B.Gate(B.MW_GATE_SOFTMAX, 8, 4, 1.0)
    l, ids, w = scores(64, 256, 1, torch.float32).contiguous(), torch.empty((64, 8), dtype=torch.int32, device=DEV), torch.empty((64, 8), device=DEV)
    dl = torch.empty_like(l)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx.mw_route(gate, l, None, ids, w)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.mw_route(gate, l, None, ids, w)
            ctx.mw_route_backward(gate, l, ids, w, dl)
    for seed in range(3):
        l.copy_(scores(64, 256, 50 + seed, torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        want_ids, want = P.route(l.cpu().numpy(), None, 8, P.SOFTMAX, 8, 4)
        np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
        d, size = P.route_backward(l.cpu().numpy(), want_ids, w.cpu().numpy(), P.SOFTMAX)
        assert (np.abs(dl.cpu().numpy() - d) <= 128 * U * size + TINY).all()


def test_refusals():
    l, ids, w = scores(4, 64, 1, torch.float32), torch.empty((4, 8), dtype=torch.int32, device=DEV), torch.empty((4, 8), device=DEV)
    ctx = make_ctx(64, 8, 4)

    def refused(status, call, *args):
        with pytest.raises(B.MwError) as e:
            call(*args)
        assert e.value.status == status

    for gate in (B.Gate(3), B.Gate(-1), B.Gate(0, 0), B.Gate(0, 5), B.Gate(0, 8, 9), B.Gate(0, 8, 0), B.Gate(0, 1, 1, float("inf")), B.Gate(0, 1, 1, float("nan"))):
        refused(B.MW_ERR_INVALID_ARG, ctx.mw_route, gate, l, None, ids, w)
        refused(B.MW_ERR_INVALID_ARG, ctx.mw_route_backward, gate, l, ids, w, l)
    many = scores(5, 64, 1, torch.float32)
    refused(B.MW_ERR_CAPACITY, ctx.mw_route, B.Gate(0), many, None, torch.empty((5, 8), dtype=torch.int32, device=DEV), torch.empty((5, 8), device=DEV))
    big = make_ctx(2048, 8, 4)
    refused(B.MW_ERR_UNSUPPORTED, big.mw_route, B.Gate(0), scores(4, 2048, 1, torch.float32), None, ids, w)
    refused(B.MW_ERR_UNSUPPORTED, make_ctx(256, 8, 4).mw_route, B.Gate(0, 128), scores(4, 256, 1, torch.float32), None, ids, w)
    for bad in (l.double(), l[:, :63], l.t(), l[0]):
        with pytest.raises((ValueError, IndexError)):
            ctx.mw_route(B.Gate(0), bad, None, ids, w)
    with pytest.raises(ValueError):
        ctx.mw_route(B.Gate(0), l, l[0].double(), ids, w)
    with pytest.raises(ValueError):
        ctx.mw_route(B.Gate(0), l, None, ids.long(), w)
    with pytest.raises(ValueError):
        ctx.mw_route_backward(B.Gate(0), l, ids, w, l.bfloat16())
    calls = B._native()
    args = [ctx._h, B.Gate(0).address, l, 0, 64, None, 4, ids, w, 0]
    for at, bad in ((1, 0), (2, None), (3, 2), (4, 63), (6, -1), (7, None), (8, None)):
        assert calls.mw_route(*(args[:at] + [bad] + args[at + 1:])) == B.MW_ERR_INVALID_ARG
    ctx.mw_route(B.Gate(0), l[:0], None, ids[:0], w[:0])          # no tokens: nothing to do
