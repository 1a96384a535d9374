"""Gates that take experts by their share plus a bias (MW_GATE_BY_SHARE), against the definition in 64 bits.

A share is rounded in fp32: the exponential's argument is off by at most 2^-24 of 20, the rest by a few 2^-24, the addition of the bias and a
group's sum by 2^-24 of values below 4 each.  Choices whose 64-bit scores are 2^-18 apart are therefore the same; tokens with a closer call at
a place that decides are left out, and are few."""
import os

import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, U, GAP = "cuda:0", 2.0 ** -24, 2.0 ** -18


def taken(l, bias, top_k, n_groups, kept, score):
    """(ids of one token, the smallest distance of two scores whose order matters)."""
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, P.BIG)).astype(np.float64)
    if score == P.SIGMOID_TOPK:
        with np.errstate(over="ignore"):
            share = 1.0 / (1.0 + np.exp(-l))
    else:
        v = np.exp(l - max(l.max(), -float(P.BIG)))
        share = v / v.sum() if v.sum() > 0 else v
    s = share + (0.0 if bias is None else bias.astype(np.float64))
    s[np.isneginf(l) | np.isnan(s)] = -np.inf
    s, gap, per = np.minimum(s, float(P.BIG)), np.inf, len(l) // n_groups
    if n_groups > 1:
        groups = -np.sort(-s.reshape(n_groups, per), 1)
        two = np.where(np.isneginf(groups[:, 1]), groups[:, 0], groups[:, 0] + groups[:, 1]) if per > 1 and score == P.SIGMOID_TOPK else groups[:, 0]
        order = sorted(range(n_groups), key=lambda g: (-two[g], g))
        if kept < n_groups and not np.isneginf(two[order[kept]]):
            gap = min(gap, two[order[kept - 1]] - two[order[kept]])
        for g in order[kept:]:
            s[g * per:(g + 1) * per] = -np.inf
    order = [e for e in np.argsort(-s, kind="stable") if not np.isneginf(s[e])]
    gap = min([gap] + [s[a] - s[b] for a, b in zip(order[:top_k], order[1:top_k + 1])])
    ids = [int(e) for e in order[:top_k]]
    return ids + [-1] * (top_k - len(ids)), gap


def route(gate, l, bias, K):
    ctx = B.Context(1, l.shape[1], K, 0, 8, B.MW_ROW_BF16, len(l), 0, np.zeros(l.shape[1], dtype=np.int32))
    ids, w = torch.full((len(l), K), -77, dtype=torch.int32, device=DEV), torch.full((len(l), K), -77.0, device=DEV)
    ctx.mw_route(gate, l, bias, ids, w)
    torch.cuda.synchronize()
    ctx.close()
    return ids.cpu().numpy(), w.cpu().numpy()


def check(l, bias, K, score, G, kept, few=0.1):
    ids, w = route(B.Gate(score, G, kept, 2.5, by_share=True), l, bias, K)
    host = l.float().cpu().numpy()
    want = [taken(row, None if bias is None else bias.cpu().numpy(), K, G, kept, score) for row in host]
    clear = np.array([gap > GAP for _, gap in want])
    assert clear.mean() >= 1 - few
    np.testing.assert_array_equal(ids[clear], np.array([i for i, _ in want], dtype=np.int32).reshape(-1, K)[clear])
    shares = np.array([P.shares(P.clean(row), i, score)[0] * 2.5 for row, i in zip(host, ids)])       # the weights of what was taken, without the bias
    assert (np.abs(w - shares) <= 64 * U * np.abs(shares) + 2.0 ** -126).all()
    return ids


SHAPES = [(1, 1, 1, 1, 1), (5, 16, 2, 4, 2), (7, 60, 4, 1, 1), (64, 64, 8, 8, 4), (9, 65, 5, 1, 1), (9, 160, 6, 8, 3), (200, 256, 8, 8, 4), (10, 256, 8, 64, 8),
          (6, 1000, 20, 1, 1), (5, 1024, 8, 2, 1), (4, 6, 3, 6, 4)]


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
@pytest.mark.parametrize("T,E,K,G,kept", SHAPES)
def test_ids_and_weights(T, E, K, G, kept, score):
    g = torch.Generator().manual_seed(T + E + score)
    for dtype, with_bias in ((torch.float32, False), (torch.float32, True), (torch.bfloat16, True)):
        # (every value once a row: bf16 scores would be equal in pairs, softmax shares of a thousand experts lie close together)
        l = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() * (8.0 / E) - 4.0
        l = torch.randn((T, E), generator=g) if dtype == torch.float32 else l.to(dtype)
        bias = (torch.randn(E, generator=g) * 0.1).to(DEV) if with_bias else None
        check(l.to(DEV), bias, K, score, G, kept, few=0.5)


def test_it_is_another_choice_than_by_score():
    """Scores and biases of a balanced gate: by score + bias nearly every token would get other experts."""
    g = torch.Generator().manual_seed(1)
    l, bias = torch.randn((300, 256), generator=g).to(DEV), (torch.randn(256, generator=g) * 0.1).to(DEV)
    ids = check(l, bias, 8, P.SIGMOID_TOPK, 8, 4)
    other, _ = route(B.Gate(P.SIGMOID_TOPK, 8, 4, 2.5), l, bias, 8)
    assert (np.sort(ids, 1) != np.sort(other, 1)).any(1).mean() > 0.9


@pytest.mark.parametrize("score", [P.SOFTMAX, P.SOFTMAX_TOPK, P.SIGMOID_TOPK])
@pytest.mark.parametrize("G,kept", [(1, 1), (8, 3)])
def test_masked_experts_and_values_that_are_no_numbers(score, G, kept):
    """A masked expert is not taken and does not count in its group, whatever the bias; nor is one whose bias is -inf or not a number."""
    inf, nan = float("inf"), float("nan")
    g = torch.Generator().manual_seed(5)
    l = torch.randn((12, 64), generator=g)
    l[0], l[1], l[2, 3:], l[3, ::2] = -inf, nan, -inf, -inf
    l[4, 7], l[5, 9], l[6, 16:] = nan, inf, -inf
    l[7, torch.arange(64) % 8 != 2] = -inf                              # one expert a group
    l[8, :] = -inf
    l[8, 60] = -3.0
    l[9, 20] = float(torch.finfo(torch.float32).min)
    bias = torch.randn(64, generator=g) * 0.5 - 1.0                     # (shares plus bias below 0: the masked are not ahead)
    check(l.to(DEV), None, 8, score, G, kept, few=0.5)
    check(l.to(DEV), bias.to(DEV), 8, score, G, kept, few=0.5)
    ids, _ = route(B.Gate(score, G, kept, by_share=True), l.to(DEV), bias.to(DEV), 8)
    assert ((ids[:, 0] >= 0) == ~(torch.isneginf(l) | torch.isnan(l)).all(1).numpy()).all()
    bias[10:20], bias[30] = -inf, nan
    check(l.to(DEV), bias.to(DEV), 8, score, G, kept, few=0.5)


def test_the_layer_and_the_gradient_take_such_gates():
    g = torch.Generator().manual_seed(7)
    T, E, K, H, I = 20, 16, 4, 64, 32
    up, down, x = ((torch.randn(s, generator=g) * s[-1] ** -0.5).bfloat16() for s in ((E, 2, I, H), (E, H, I), (T, H)))
    l, bias, dw = torch.randn((T, E), generator=g), torch.randn(E, generator=g) * 0.3, torch.randn((T, K), generator=g)
    ctx = B.Context(1, E, K, 0, H, B.MW_ROW_BF16, T, 0, np.zeros(E, dtype=np.int32))
    experts, gate = B.Experts(up.to(DEV), down.to(DEV)), B.Gate(B.MW_GATE_SIGMOID_TOPK, 4, 2, 2.5, by_share=True)
    ids, w, d = torch.empty((T, K), dtype=torch.int32, device=DEV), torch.empty((T, K), device=DEV), torch.empty((T, E), device=DEV)
    out = torch.empty((T, H), dtype=torch.bfloat16, device=DEV)
    ctx.mw_moe_layer(gate, l.to(DEV), bias.to(DEV), experts, x.to(DEV), ids, w, out, ctx.moe_workspace(experts, T))
    ctx.mw_route_backward(gate, l.to(DEV), ids, dw.to(DEV), d)
    torch.cuda.synchronize()
    ids, w = ids.cpu().numpy(), w.cpu().numpy()
    want = [taken(row, bias.numpy(), K, 4, 2, P.SIGMOID_TOPK) for row in l.numpy()]
    assert all(gap <= GAP or list(got) == i for got, (i, gap) in zip(ids, want))
    want, off = P.layer(x.double().numpy(), ids, w, up.double().numpy(), down.double().numpy(), {i: i for i in range(E)}, 128 * U)
    assert (np.abs(out.float().cpu().numpy() - want) <= off + 2.0 ** -8 * np.abs(want)).all()
    want, size = P.route_backward(l.numpy(), ids, dw.numpy(), P.SIGMOID_TOPK, 2.5)
    assert (np.abs(d.cpu().numpy() - want) <= 128 * U * size + 2.0 ** -126).all()
    ctx.close()


def test_refusals():
    l, ids, w = torch.zeros((4, 64), device=DEV), torch.empty((4, 8), dtype=torch.int32, device=DEV), torch.empty((4, 8), device=DEV)
    ctx = B.Context(1, 64, 8, 0, 8, B.MW_ROW_BF16, 4, 0, np.zeros(64, dtype=np.int32))
    for score in (3, 0x20, 0x12 | 0x20, 4):
        with pytest.raises(B.MwError) as e:
            ctx.mw_route(B.Gate(score, by_share=True), l, None, ids, w)
        assert e.value.status == B.MW_ERR_INVALID_ARG
    ctx.close()


def test_the_constant_is_the_headers():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mw.h")).read()
    line, = [l.split() for l in text.splitlines() if l.startswith("#define MW_GATE_BY_SHARE ")]
    assert int(line[2], 0) == B.MW_GATE_BY_SHARE


def test_the_example_with_such_a_gate():
    import importlib.util
    spec = importlib.util.spec_from_file_location("moe_block", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    block = module.Block(n_ranks=4, rank=1, n_experts=16, top_k=4, hidden=256, inter=128, adapter_rank=8, n_adapters=3, max_tokens=64, by_share=True)
    g = torch.Generator().manual_seed(1)
    x, requests = torch.randn((40, 256), generator=g).bfloat16().to(DEV), torch.randint(-1, 3, (40,), generator=g).int().to(DEV)
    _, ids, _ = block.decode(x, requests)
    scores = block.route(block.project(x, requests))[0].cpu().numpy()
    want = [taken(row, np.zeros(16), 4, 4, 2, P.SIGMOID_TOPK) for row in scores]
    assert all(gap <= GAP or list(got) == i for got, (i, gap) in zip(ids.cpu().numpy(), want))
    send, stats = block.prefill(x, requests)
    assert int(stats["n_rows"]) == 40 and int(stats["error_flags"]) == 0
