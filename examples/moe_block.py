"""A rank's mixture-of-experts block around the dispatch.

decode():   a few tokens of several requests, with each request's adapter on a shared projection and the rank's experts in place (no dispatch)
prefill():  the same gate in front of a dispatch: its ids go straight into the plan
receive():  what of a dispatch arrives here, rows in the order of this rank's experts; run_experts(): their blocks over these rows and the way back
training(): one step of the adapters and the gate's scores
training_experts(): gradients of the experts, of the rows that arrived, and through their gate weights of the gate's scores

Run on one GPU: python examples/moe_block.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_22428_amd import binding as B  # noqa: E402


class Block:
    """The weights of one block on rank `rank` of `n_ranks`, random; the buffers that its calls keep using.  by_share: the gate of a model whose
    bias stands beside sigmoids, else beside scores; another choice of experts, so it has to be the one the weights were trained with."""

    def __init__(self, n_ranks=8, rank=0, n_experts=64, top_k=8, hidden=4096, inter=1024, adapter_rank=16, n_adapters=12, max_tokens=256, seed=1,
                 device="cuda:0", by_share=False):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=g, device=device, dtype=torch.bfloat16) * shape[-1] ** -0.5

        place = (np.arange(n_experts) * n_ranks // n_experts).astype(np.int32)
        n_local = int((place == rank).sum())
        self.ctx = B.Context(n_ranks, n_experts, top_k, rank, hidden, B.MW_ROW_BF16, max_tokens, max_tokens, place, device=device)
        self.gate = B.Gate(B.MW_GATE_SIGMOID_TOPK, n_groups=n_ranks, kept_groups=max(1, n_ranks // 2), scale=2.5, by_share=by_share)
        self.gate_weight, self.gate_bias = normal(n_experts, hidden), torch.zeros(n_experts, device=device)
        self.experts = B.Experts(normal(n_local, 2, inter, hidden), normal(n_local, hidden, inter))
        self.projection = normal(hidden, hidden)
        self.adapters = B.Adapters(normal(n_adapters, adapter_rank, hidden), normal(n_adapters, hidden, adapter_rank),
                                   torch.full((n_adapters,), 2.0, device=device))
        self.layer_workspace = self.ctx.moe_workspace(self.experts, max_tokens)
        self.adapter_workspace = self.adapters.workspace(max_tokens)
        self.top_k, self.hidden, self.inter, self.device, self.rank = top_k, hidden, inter, device, rank
        self.first_expert, self.n_local, self.room = int((place < rank).sum()), n_local, max_tokens * min(top_k, n_local)
        self.ffn_workspace = self.ctx.ffn_workspace(self.experts, self.room, backward=True)

    def experts_in_codes(self):
        """The same experts in 8-bit codes; an output channel of a matrix is a row to quantize."""
        made = []
        for w in self.experts._held[:2]:
            codes, scales = torch.empty(w.shape, dtype=torch.int8, device=self.device), torch.empty(w.shape[:-1], device=self.device)
            B.mw_quantize_rows(w.flatten(0, -2), codes.flatten(0, -2), scales.flatten())
            made.append((codes, scales))
        return B.Experts(made[0][0], made[1][0], made[0][1], made[1][1])

    def project(self, x, adapter_ids, keep_h=False):
        """The shared projection and every row's own adapter beside it; in place on the projection's output."""
        y = x @ self.projection.t()
        h = torch.empty((x.shape[0], self.adapters.rank), device=self.device) if keep_h else None
        self.adapters.mw_adapt(x, adapter_ids, y, y, self.adapter_workspace, h)
        return (y, h) if keep_h else y

    def route(self, x):
        scores = x.float() @ self.gate_weight.float().t()
        ids = torch.empty((x.shape[0], self.top_k), dtype=torch.int32, device=self.device)
        weights = torch.empty((x.shape[0], self.top_k), device=self.device)
        return scores, ids, weights

    def decode(self, x, adapter_ids):
        """(output of this rank's experts, ids, weights); ranks add their outputs up (an all-reduce, where there are several)."""
        y = self.project(x, adapter_ids)
        scores, ids, weights = self.route(y)
        out = torch.empty_like(y)
        self.ctx.mw_moe_layer(self.gate, scores, self.gate_bias, self.experts, y, ids, weights, out, self.layer_workspace)
        return out, ids, weights

    def prefill(self, x, adapter_ids):
        """The send side of a dispatch: projection, gate, plan and pack.  Returns the packed rows and the statistics."""
        y = self.project(x, adapter_ids)
        scores, ids, weights = self.route(y)
        send = B.SendBuffers(self.ctx, x.shape[0])
        self.ctx.mw_route(self.gate, scores, self.gate_bias, ids, weights)
        self.ctx.mw_plan(ids, send.mask, send.perm, send.desc, send.stats)
        self.ctx.mw_pack(y, None, ids, send.perm, send.stats, send.packed, send.row_src_token, send.row_topk)
        return send, self.ctx.mw_get_send_stats(send.stats)

    def receive(self, send, n_tokens, ids, weights):
        """What of this rank's tokens goes to its own experts (the other ranks' rows come the same way, one region a rank): the unpacked rows, and every row's gate weight."""
        ctx, n = self.ctx, max(n_tokens, 1)
        region = dict(desc=torch.zeros((n, B.DESC_BYTES), dtype=torch.uint8, device=self.device), rows=torch.zeros((n, ctx.row_stride), dtype=torch.uint8, device=self.device),
                      row_src_token=torch.zeros((n,), dtype=torch.int32, device=self.device), row_topk=torch.zeros((n, self.top_k), dtype=torch.int32, device=self.device))
        counts = torch.zeros(2, dtype=torch.int32, device=self.device)
        ctx.mw_sim_deliver(send.desc, send.stats, n_tokens, send.packed, send.row_src_token, send.row_topk, self.rank, region["desc"], region["rows"], region["row_src_token"],
                           region["row_topk"], counts)
        region["n_desc"], region["n_rows"] = counts.tolist()
        recv = B.RecvBuffers(ctx, self.room)
        recv.table = B.peers_table([region], self.device)
        ctx.mw_unpack(recv.table, 1, recv.out_rows, recv.out_scales, self.room, recv.out_src_peer, recv.out_src_token, recv.expert_offsets, recv.stats)
        recv.rows, recv.n_back, recv.n_rows = recv.out_rows.view(torch.bfloat16), region["n_rows"], int(ctx.mw_get_recv_stats(recv.stats)["n_out_rows"])
        # a row's weight is that of its token for its expert, and a place in the weights
        place = torch.arange(self.room, device=self.device)
        expert = self.first_expert + torch.searchsorted(recv.expert_offsets[1:], place, right=True)
        recv.token = recv.out_src_token.long().clamp(min=0)
        recv.hit = (ids[recv.token] == expert[:, None]) & (place < recv.n_rows)[:, None]
        recv.row_weights = (weights[recv.token] * recv.hit).sum(1)
        return recv

    def run_experts(self, recv, experts=None, keep=False):
        """The experts' blocks over the rows that arrived, and what goes back: a summed row for every row received.  With keep also the gate and up values."""
        experts = experts or self.experts
        y, back = torch.zeros_like(recv.rows), torch.zeros((max(recv.n_back, 1), self.hidden), dtype=torch.bfloat16, device=self.device)
        kept = torch.empty((self.room, 2, self.inter), dtype=torch.bfloat16, device=self.device) if keep else None
        self.ctx.mw_ffn(experts, recv.rows, recv.expert_offsets, y, self.ffn_workspace, recv.row_weights, kept)
        self.ctx.mw_combine_gather(1, y, self.room, back, back.shape[0])
        return (y, back[:recv.n_back], kept) if keep else (y, back[:recv.n_back])

    def training_experts(self, recv, kept, d_y, scores, ids):
        """For the gradient of the experts' rows: gradients of the rows that arrived, of this rank's experts, and of the gate's scores."""
        gate_up, down = self.experts._held[:2]
        d_rows, d_gate_up, d_down = torch.zeros_like(recv.rows), torch.empty_like(gate_up), torch.empty_like(down)
        d_row_weights = torch.zeros((self.room,), device=self.device)
        self.ctx.mw_ffn_backward(self.experts, recv.rows, recv.expert_offsets, kept, d_y, d_rows, d_gate_up, d_down, self.ffn_workspace, recv.row_weights, d_row_weights)
        d_weights = torch.zeros(ids.shape, device=self.device).index_add_(0, recv.token, d_row_weights[:, None] * recv.hit)
        d_scores = torch.empty_like(scores)
        self.ctx.mw_route_backward(self.gate, scores, ids, d_weights, d_scores)
        return d_rows, d_gate_up, d_down, d_weights, d_scores

    def training(self, x, adapter_ids, d_y, d_weights):
        """Gradients of the input, of both factors of every adapter, and of the gate's scores, for given gradients of the projection's output and
        of the gate's weights."""
        y, h = self.project(x, adapter_ids, keep_h=True)
        scores, ids, weights = self.route(y)
        self.ctx.mw_route(self.gate, scores, self.gate_bias, ids, weights)
        d_scores = torch.empty_like(scores)
        self.ctx.mw_route_backward(self.gate, scores, ids, d_weights, d_scores)
        d_y = d_y + (d_scores @ self.gate_weight.float()).bfloat16()
        d_x, d_a, d_b = d_y @ self.projection, torch.empty_like(self.adapters.a), torch.empty_like(self.adapters.b)
        self.adapters.mw_adapt_backward(x, adapter_ids, h, d_y, d_x, d_x, d_a, d_b, self.adapter_workspace)
        return d_x, d_a, d_b, d_scores


def main():
    block, g = Block(), torch.Generator(device="cuda:0")
    g.manual_seed(2)
    for n in (1, 64, 256):
        x = torch.randn((n, block.hidden), generator=g, device="cuda:0", dtype=torch.bfloat16)
        requests = torch.randint(-1, block.adapters.n, (n,), generator=g, device="cuda:0").int()
        out, ids, _ = block.decode(x, requests)
        send, stats = block.prefill(x, requests)
        d = block.training(x, requests, torch.randn(x.shape, generator=g, device="cuda:0", dtype=torch.bfloat16),
                           torch.randn(ids.shape, generator=g, device="cuda:0"))
        scores, ids, weights = block.route(block.project(x, requests))
        block.ctx.mw_route(block.gate, scores, block.gate_bias, ids, weights)
        recv = block.receive(send, n, ids, weights)
        y, back, kept = block.run_experts(recv, keep=True)
        e = block.training_experts(recv, kept, torch.randn(y.shape, generator=g, device="cuda:0", dtype=torch.bfloat16), scores, ids)
        coded, _ = block.run_experts(recv, block.experts_in_codes())
        torch.cuda.synchronize()
        print("    %d rows here, |y| %.3f, in codes %.3f, |back| %.3f, |d_rows| %.1f, |d_gate_up| %.1f, |d_down| %.1f, |d_scores| %.3f" % (
            recv.n_rows, y.float().norm(), coded.float().norm(), back.float().norm(), *(t.float().norm() for t in (e[0], e[1], e[2], e[4]))), flush=True)
        print("%3d tokens: |out| %.3f, %d rows packed for %d ranks, |d_x| %.1f, |d_a| %.1f, |d_b| %.1f" % (
            n, out.float().norm(), stats["n_rows"], (np.asarray(stats["rows_per_dest"]) > 0).sum(), *(t.float().norm() for t in d[:3])), flush=True)


if __name__ == "__main__":
    main()
