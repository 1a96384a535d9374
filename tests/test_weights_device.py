"""Experts and adapters whose arrays are not on the device that a call runs on are refused before the library is called.  No GPU needed."""
import pytest
import torch

from paper_2605_22428_amd import binding as B


class Calls:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError("%s was called" % name)
        return call


@pytest.mark.parametrize("current", [0, 1])
def test_adapters_of_another_device(monkeypatch, current):
    monkeypatch.setattr(B, "_native", Calls)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    a, b, x, y = (torch.zeros(s, dtype=torch.bfloat16) for s in ((2, 8, 16), (2, 24, 8), (3, 16), (3, 24)))
    adapters, ids, h = B.Adapters(a, b), torch.zeros(3, dtype=torch.int32), torch.zeros((3, 8))
    ws = torch.zeros(1024, dtype=torch.uint8)
    for device in (torch.device("cpu"), torch.device("cuda", 1 - current)):
        adapters.device = device
        for call, name in ((lambda: adapters.mw_adapt(x, ids, None, y, ws), "mw_adapt"), (lambda: adapters.mw_adapt_backward(x, ids, h, y, None, x, a, b, ws), "mw_adapt_backward")):
            with pytest.raises(B.MwError, match=name + ": arrays on") as e:
                call()
            assert e.value.status == B.MW_ERR_INVALID_ARG


def test_experts_of_another_device(monkeypatch):
    monkeypatch.setattr(B, "_native", Calls)
    ctx = B.Context.__new__(B.Context)
    ctx._h, ctx.n_experts, ctx.top_k, ctx.n_local, ctx.hidden = None, 4, 2, 1, 16
    ctx.workspace = torch.empty(0, device="meta")
    experts = B.Experts(torch.zeros((1, 2, 8, 16), dtype=torch.bfloat16), torch.zeros((1, 16, 8), dtype=torch.bfloat16))
    x, ids, w, ws = torch.zeros((3, 16), dtype=torch.bfloat16), torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2)), torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(ValueError, match="weights on cpu"):
        ctx.mw_moe_layer(None, None, None, experts, x, ids, w, torch.empty_like(x), ws)
