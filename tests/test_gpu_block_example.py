"""examples/moe_block.py: gate, experts and adapters together as a rank uses them, against the plain forms of each on the values that
really went into it."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import plain_block as P

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GAMMA = 300 * 2.0 ** -24


def example():
    spec = importlib.util.spec_from_file_location("moe_block", os.path.join(ROOT, "examples", "moe_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def near(got, want, off):
    got = got.float().cpu().numpy()
    assert (np.abs(got - want) <= off + 2.0 ** -8 * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("T", [1, 16, 40])
def test_the_block_as_a_whole(T):
    block = example().Block(n_ranks=4, rank=1, n_experts=16, top_k=4, hidden=256, inter=128, adapter_rank=8, n_adapters=3, max_tokens=64)
    g = torch.Generator().manual_seed(T)
    x, requests = torch.randn((T, 256), generator=g).bfloat16(), torch.randint(-1, 3, (T,), generator=g).int()
    a, b, scale = (t.double().cpu().numpy() for t in block.adapters._held)
    base = (x.cuda() @ block.projection.t())
    y, h = block.project(x.cuda(), requests.cuda(), keep_h=True)
    want, want_h, off, off_h = P.adapt(x.double().numpy(), requests.numpy(), base.double().cpu().numpy(), a, b, scale, GAMMA)
    near(y, want, off)
    assert (np.abs(h.cpu().numpy() - want_h) <= off_h + 1e-30).all()

    out, ids, weights = block.decode(x.cuda(), requests.cuda())
    scores = block.route(y)[0].cpu().numpy()
    want_ids, want_w = P.route(scores, np.zeros(16, dtype=np.float32), 4, P.SIGMOID_TOPK, 4, 2, 2.5)
    np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
    up, down = (t.double().cpu().numpy() for t in block.experts._held[:2])
    want, off = P.layer(y.double().cpu().numpy(), want_ids, weights.cpu().numpy(), up, down, {4 + i: i for i in range(4)}, GAMMA)
    near(out, want, off)

    send, stats = block.prefill(x.cuda(), requests.cuda())
    assert int(stats["n_rows"]) == T and int(stats["error_flags"]) == 0
    perm = send.perm.cpu().numpy()[:T]
    packed = send.packed.view(torch.uint8).reshape(-1)[:T * 512].view(torch.bfloat16).reshape(T, 256)
    assert torch.equal(packed.cpu(), y.cpu()[torch.from_numpy(perm).long()])

    d_y, d_w = torch.randn((T, 256), generator=g).bfloat16(), torch.randn((T, 4), generator=g)
    d_x, d_a, d_b, d_scores = block.training(x.cuda(), requests.cuda(), d_y.cuda(), d_w.cuda())
    want_s, size = P.route_backward(scores, want_ids, d_w.numpy(), P.SIGMOID_TOPK, 2.5)
    assert (np.abs(d_scores.cpu().numpy() - want_s) <= 128 * 2.0 ** -24 * size + 2.0 ** -126).all()
    through = d_y.cuda() + (d_scores @ block.gate_weight.float()).bfloat16()
    want = P.adapt_backward(x.double().numpy(), requests.numpy(), h.double().cpu().numpy(), through.double().cpu().numpy(),
                            (through @ block.projection).double().cpu().numpy(), a, b, scale, GAMMA)
    for got, (w, off) in zip((d_x, d_a, d_b), want):
        near(got, w, off)


def test_the_example_runs(capsys):
    example().main()
    assert capsys.readouterr().out.count("tokens:") == 3
