"""Gate, dispatch, experts over the rows that arrive, the way back, and their backward pass as examples/moe_block.py runs them together, against the plain forms of each on the
values that really went into it."""
import numpy as np
import pytest
import torch

import plain_block as G
import plain_experts as P
from test_gpu_block_example import example
from test_gpu_ffn import host, near

pytestmark = pytest.mark.gpu


def run(T, seed):
    block = example().Block(n_ranks=4, rank=1, n_experts=16, top_k=4, hidden=256, inter=144, adapter_rank=8, n_adapters=3, max_tokens=96, seed=seed)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, 256), generator=g).bfloat16().cuda()
    none = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    send, _ = block.prefill(x, none)
    sent = block.project(x, none)
    scores, ids, weights = block.route(sent)
    block.ctx.mw_route(block.gate, scores, block.gate_bias, ids, weights)
    return block, g, sent, scores, ids, weights, block.receive(send, T, ids, weights)


@pytest.mark.parametrize("T,seed", [(1, 1), (1, 5), (16, 2), (96, 3)])
def test_the_experts_behind_a_dispatch(T, seed):
    block, g, sent, scores, ids, weights, recv = run(T, seed)
    ids_h, weights_h, offsets = ids.cpu().numpy(), weights.cpu().numpy(), recv.expert_offsets.cpu().numpy()
    # every (token, local expert) pair is a row, in the order of experts and tokens, with its weight
    pairs = [(e, t) for e in range(4) for t in range(T) if 4 + e in ids_h[t]]
    assert recv.n_rows == len(pairs) == offsets[-1] and (np.diff(offsets) == [sum(p[0] == e for p in pairs) for e in range(4)]).all()
    for r, (e, t) in enumerate(pairs):
        assert torch.equal(recv.rows[r], sent[t]) and float(recv.row_weights[r]) == weights_h[t][ids_h[t] == 4 + e].sum()
    y, back, kept = block.run_experts(recv, keep=True)
    gate_up, down = (host(t) for t in block.experts._held[:2])
    d_y = torch.randn(y.shape, generator=g).bfloat16().cuda()
    d_rows, d_gate_up, d_down, d_weights, d_scores = block.training_experts(recv, kept, d_y, scores, ids)
    want_d_weights, off_d_weights = np.zeros((T, 4)), np.zeros((T, 4))
    for e in range(4):
        at = slice(offsets[e], offsets[e + 1])
        if at.start == at.stop:
            assert (d_gate_up[e] == 0).all() and (d_down[e] == 0).all()
            continue
        w = host(recv.row_weights[at])
        (want, off), (want_kept, off_kept) = P.block(host(recv.rows[at]), gate_up[e], down[e], w)
        near(y[at], want, off)
        near(kept[at], want_kept, off_kept)
        grads = P.block_backward(host(recv.rows[at]), gate_up[e], down[e], w, host(kept[at]), host(d_y[at]))
        for got, (v, o) in zip((d_rows[at], d_gate_up[e], d_down[e]), grads):
            near(got, v, o)
        for (v, o), (_, t) in zip(zip(*grads[3]), pairs[at]):
            want_d_weights[t, ids_h[t] == 4 + e] += v
            off_d_weights[t, ids_h[t] == 4 + e] += o + 2 * P.U * abs(v)
    near(d_weights, want_d_weights, off_d_weights, P.U)
    # the way back: a token's rows summed in single precision, one row for every token that came
    first = {}
    for r, (e, t) in enumerate(pairs):
        first.setdefault(t, []).append(r)
    assert recv.n_back == len(first)
    sums = sorted(tuple(host(y[rows].float().sum(0).bfloat16())) if len(rows) > 2 else tuple(host((y[rows[0]].float() + y[rows[1]].float()).bfloat16() if len(rows) == 2 else y[rows[0]]))
                  for rows in first.values() if len(rows) <= 2)
    got = {tuple(host(b)) for b in back}
    assert all(s in got for s in sums)
    want, size = G.route_backward(scores.cpu().numpy(), ids_h, d_weights.cpu().numpy(), G.SIGMOID_TOPK, 2.5)
    assert (np.abs(d_scores.cpu().numpy() - want) <= 128 * P.U * size + 2.0 ** -126).all()


def test_experts_in_codes_are_near_their_originals():
    """The codes of experts and of rows are off by half a step each, a 254th of the largest value of a channel or a row."""
    block, _, _, _, _, _, recv = run(96, 7)
    coded = block.experts_in_codes()
    for (w, c, s) in zip(block.experts._held[:2], coded._held[:2], coded._held[2:]):
        want, scales = P.codes_of(host(w.flatten(0, -2)))
        np.testing.assert_array_equal(c.flatten(0, -2).cpu().numpy(), want)
        np.testing.assert_array_equal(s.flatten().cpu().numpy(), scales)
    y, _ = block.run_experts(recv)
    z, _ = block.run_experts(recv, coded)
    # largest values are about 3.5 deviations: a code is off by 3.5 / 254 / sqrt(3) deviations, four such errors (rows, weights, inner rows, weights) in a product
    assert (y - z).float().norm() <= 3 * 4 ** 0.5 * 3.5 / 254 / 3 ** 0.5 * y.float().norm()


def test_a_step_replayed_from_a_graph():
    """Experts forward, the way back and backward, captured once; rows, offsets, weights and gradients change before every replay, eager work of the same kind stands between."""
    block, g, _, _, _, _, recv = run(96, 11)
    other = run(96, 12)[-1]
    d_y = torch.zeros_like(recv.rows)
    y, kept = torch.zeros_like(recv.rows), torch.zeros((block.room, 2, block.inter), dtype=torch.bfloat16, device="cuda")
    d_rows, d_w = torch.zeros_like(recv.rows), torch.zeros(block.room, device="cuda")
    gate_up, down = block.experts._held[:2]
    d_gate_up, d_down, ws = torch.empty_like(gate_up), torch.empty_like(down), block.ctx.ffn_workspace(block.experts, block.room, True)
    coded, z = block.experts_in_codes(), torch.zeros_like(recv.rows)

    def step():
        block.ctx.mw_ffn(block.experts, recv.rows, recv.expert_offsets, y, ws, recv.row_weights, kept)
        block.ctx.mw_ffn_backward(block.experts, recv.rows, recv.expert_offsets, kept, d_y, d_rows, d_gate_up, d_down, ws, recv.row_weights, d_w)
        block.ctx.mw_ffn(coded, recv.rows, recv.expert_offsets, z, ws, recv.row_weights)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    sources = [[t.clone() for t in (r.rows, r.expert_offsets, r.row_weights)] for r in (recv, other)]
    for turn in range(4):
        for to, v in zip((recv.rows, recv.expert_offsets, recv.row_weights), sources[turn % 2]):
            to.copy_(v)
        d_y.copy_(torch.randn(d_y.shape, generator=g).bfloat16())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        n = int(recv.expert_offsets[-1])
        got = [t[:n].clone() for t in (y, kept, d_rows, d_w, z)] + [d_gate_up.clone(), d_down.clone()]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, [t[:n] for t in (y, kept, d_rows, d_w, z)] + [d_gate_up, d_down]):
            assert torch.equal(a, b)
