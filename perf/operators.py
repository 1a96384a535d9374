"""A rank's mixture-of-experts block around the dispatch, as timed cases: its gate, its experts for a few tokens, and the adapters
of many requests beside a shared projection.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a program holds before the call, run() is one
pass, work() the bytes and operations a pass cannot do without, exact() the results in 64 bits.  Where `own` is true run() makes the
library's calls, else it computes the same in elementary torch operations in 32 bits, rounded once at the end.

Kinds of cases
  route           mw_route: gate scores -> expert ids (what mw_plan takes) and gate weights
  route_backward  mw_route_backward: gradient of the gate weights -> gradient of the scores
  layer           mw_moe_layer: scores and at most 256 tokens -> the sum of their local experts' outputs
  adapt           mw_adapt: base + scale * B (A x), every row with its own adapter or none
  adapt_backward  mw_adapt_backward: gradients of the input and of every adapter

The product that makes the scores and the shared projection itself are plain matrix products and not part of these operators.
"""
import math

import numpy as np
import torch

DEV = "cuda:0"
own = False
BIG = torch.finfo(torch.float32).max
SCORES = ("softmax", "softmax_topk", "sigmoid_topk")
LARGEST_BYTES = 2.9e9


def _gate(name, kind, tokens, experts, top_k, score, groups=1, kept=1, bias=False, logits="f32", masked=0.0):
    return dict(name=name, kind=kind, tokens=tokens, experts=experts, top_k=top_k, score=score, groups=groups, kept=kept,
                bias=bias, logits=logits, masked=masked)


def _layer(name, tokens, ranks, experts, top_k, hidden, inter, weights, score="softmax_topk", groups=1, kept=1, bias=False):
    return dict(_gate(name, "layer", tokens, experts, top_k, score, groups, kept, bias), ranks=ranks, hidden=hidden, inter=inter,
                weights=weights)


def _adapt(name, kind, rows, adapters, rank, n_in, n_out, order, none=0.0, pad=0):
    return dict(name=name, kind=kind, rows=rows, adapters=adapters, rank=rank, n_in=n_in, n_out=n_out, order=order, none=none, pad=pad)


def listed():
    return [
        # the gate of a decode batch on a small job: 16 experts, top-2; a launch and its latency
        _gate("route_128tok_16e", "route", 128, 16, 2, "softmax_topk"),
        # the gate of a prefill batch: 256 experts in 8 groups of which 4 are kept, balancing bias, some experts masked
        _gate("route_8192tok_256e_groups", "route", 8192, 256, 8, "sigmoid_topk", 8, 4, True, masked=0.02),
        # training: the same batch size with scores and their gradient in bf16
        _gate("route_backward_4096tok_bf16", "route_backward", 4096, 256, 8, "softmax", logits="bf16"),
        # training, an odd number of experts and tokens
        _gate("route_backward_1000tok_60e", "route_backward", 1000, 60, 4, "sigmoid_topk", masked=0.05),
        # one token, the paper's 64 experts and top-8, the whole layer on one GPU
        _layer("layer_1tok_64e", 1, 1, 64, 8, 4096, 1024, "bf16"),
        # odd sizes: 13 tokens, hidden size no multiple of a tile
        _layer("layer_13tok_16e_odd", 13, 2, 16, 2, 2880, 1000, "bf16", "softmax"),
        # a decode batch of 64 tokens a rank of a 64-rank job, four fp8 experts on each rank, every rank has the tokens
        _layer("layer_64tok_ep64_fp8", 64, 64, 256, 8, 7168, 2048, "fp8", "sigmoid_topk", 8, 4, True),
        # the largest: 256 tokens on one of 8 ranks, 32 bf16 experts there
        _layer("layer_256tok_ep8", 256, 8, 256, 8, 7168, 2048, "bf16", "sigmoid_topk", 8, 4, True),
        # token generation for 64 requests with 24 adapters between them, some with none
        _adapt("adapt_64req_r16", "adapt", 64, 24, 16, 7168, 7168, "mixed", none=0.15),
        # prompts of 8 requests in one batch, rows of one request together
        _adapt("adapt_8192tok_r32", "adapt", 8192, 8, 32, 7168, 4096, "prompts", none=0.1),
        # a few rows of one user's adapter being trained, a view of wider rows
        _adapt("adapt_backward_333tok_r8", "adapt_backward", 333, 3, 8, 1024, 2880, "prompts", pad=64),
        # four adapters trained at once on a batch of mixed rows
        _adapt("adapt_backward_4096tok_r64", "adapt_backward", 4096, 4, 64, 4096, 4096, "mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["route", "route", "route_backward", "layer", "layer", "layer", "adapt", "adapt", "adapt_backward"])
    if kind.startswith("adapt"):
        rows = _log_int(rng, 1, 8192)
        n_in, n_out = (rng.choice([256, 328, 1024, 2048, 2880, 4096, 5120, 7168]) for _ in range(2))
        return dict(kind=kind, rows=rows, adapters=_log_int(rng, 1, 64), rank=rng.choice([8, 16, 16, 32, 64]), n_in=n_in, n_out=n_out,
                    order=rng.choice(["mixed", "prompts"]), none=rng.choice([0.0, 0.0, 0.2]), pad=rng.choice([0, 0, 8, 64]))
    experts, groups = rng.choice([(8, 1), (16, 1), (16, 4), (60, 1), (64, 8), (128, 1), (160, 8), (256, 1), (256, 8), (384, 1)])
    c = dict(kind=kind, tokens=_log_int(rng, 1, 256 if kind == "layer" else 8192), experts=experts,
             top_k=rng.choice([k for k in (1, 2, 4, 6, 8, 8, 9) if k <= experts // 2]), score=rng.choice(SCORES), groups=groups,
             kept=max(1, groups // 2), bias=rng.random() < 0.5, logits="f32", masked=0.0)
    if c["top_k"] == 1:                               # (normalised, the only choice would weigh the same whatever the scores)
        c["score"] = "softmax"
    if kind == "layer":
        c.update(ranks=rng.choice([r for r in (1, 2, 4, 8, 16, 64) if r <= experts]), hidden=rng.choice([256, 328, 1024, 2048, 2880, 4096, 7168]),
                 inter=rng.choice([256, 512, 768, 1000, 1408, 2048]), weights=rng.choice(["bf16", "fp8"]))
        if c["weights"] == "fp8":                     # rows of whole 16-byte pieces
            c["hidden"], c["inter"] = c["hidden"] // 16 * 16, c["inter"] // 16 * 16
    else:
        c.update(logits=rng.choice(["f32", "bf16"]), masked=rng.choice([0.0, 0.0, 0.03]))
    return c


def draw(rng):
    while True:
        c = _draw_once(rng)
        sizes = [v for v in c.values() if not isinstance(v, (str, float))]
        held = 3 * 2 * _local(c) * c["hidden"] * c["inter"] if c["kind"] == "layer" else 0
        if 3072 not in sizes and work(c)["bytes"] <= LARGEST_BYTES and held <= LARGEST_BYTES:
            return c


# ---- what a case consists of ----------------------------------------------------------------------
def _placement(c):
    """Rank of every expert: contiguous, as even as the counts allow."""
    return (np.arange(c["experts"], dtype=np.int64) * c["ranks"] // c["experts"]).astype(np.int32)


def _local(c):
    return int((_placement(c) == 0).sum())            # this rank is rank 0: experts 0 .. _local - 1


def _weight_bytes(c, rows, cols):
    blocks = -(-rows // 128) * -(-cols // 128)
    return 2.0 * rows * cols if c["weights"] == "bf16" else 1.0 * rows * cols + 4.0 * blocks


def work(case):
    c = case
    if c["kind"].startswith("adapt"):
        t, r, m, o = c["rows"] * (1 - c["none"]), c["rank"], c["n_in"], c["n_out"]
        n = min(c["adapters"], c["rows"]) if c["order"] == "prompts" else c["adapters"] * (1 - (1 - 1 / c["adapters"]) ** t)
        params = 2.0 * n * r * (m + o)
        if c["kind"] == "adapt":
            return {"bytes": params + 2.0 * t * m + 4.0 * c["rows"] * o + 4.0 * c["rows"], "flops": 2.0 * t * r * (m + o)}
        grads = 2.0 * c["adapters"] * r * (m + o)
        return {"bytes": params + grads + 2.0 * t * (m + o) + 4.0 * c["rows"] * m + 4.0 * t * r + 4.0 * c["rows"], "flops": 4.0 * t * r * (m + o)}
    t, e, k = c["tokens"], c["experts"], c["top_k"]
    scores = float(t * e * (2 if c["logits"] == "bf16" else 4))
    if c["kind"] == "route":
        return {"bytes": scores + 8.0 * t * k, "flops": 8.0 * t * e}
    if c["kind"] == "route_backward":
        return {"bytes": 2 * scores + 8.0 * t * k, "flops": 8.0 * t * e}
    h, i, n = c["hidden"], c["inter"], _local(c)
    hit = n * (1 - (1 - k / e) ** t)
    expert = 2 * _weight_bytes(c, i, h) + _weight_bytes(c, h, i)
    return {"bytes": hit * expert + 4.0 * t * h + scores + 8.0 * t * k, "flops": 6.0 * t * k * n / e * h * i}


# ---- inputs -----------------------------------------------------------------------------------------
def _generator(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + tag) % (1 << 62))
    return g


def _normal(seed, tag, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_generator(seed, tag), dtype=dtype, device=DEV).mul_(std)


def _rows(seed, tag, n, width, pad):
    """n rows of N(0, 1) values; with a pad a view of wider rows."""
    return _normal(seed, tag, (n, width + pad))[:, :width]


def _fp8(w):
    """[..., rows, cols] -> e4m3 codes and one scale per 128 x 128 block (blocks at the edges are smaller)."""
    rows, cols = w.shape[-2:]
    full = torch.nn.functional.pad(w.float(), (0, -cols % 128, 0, -rows % 128))
    blocks = full.unflatten(-1, (-1, 128)).unflatten(-3, (-1, 128))
    scale = blocks.abs().amax((-3, -1)).clamp_(min=1e-6) / 448.0
    codes = (blocks / scale[..., :, None, :, None]).clamp_(-448, 448).flatten(-2).flatten(-3, -2)[..., :rows, :cols]
    return codes.to(torch.float8_e4m3fn).contiguous(), scale.contiguous()


def _wide(codes, scale, dtype=torch.float32):
    """The weights that codes and scales stand for."""
    rows, cols = codes.shape[-2:]
    return codes.to(dtype) * scale.to(dtype).repeat_interleave(128, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :cols]


def _adapter_ids(c, seed):
    g, n, t = _generator(seed, 3), c["adapters"], c["rows"]
    ids = torch.randint(0, n, (t,), generator=g, device=DEV)
    if c["order"] == "prompts":                       # rows of one request together, requests of uneven lengths
        ids = ids.sort().values if n < t else ids
        ids = torch.randperm(n, generator=g, device=DEV)[ids]
    if c["none"]:
        ids = torch.where(torch.rand((t,), generator=g, device=DEV) < c["none"], -1, ids)
    return ids.int()


class _State:
    pass


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    if c["kind"].startswith("adapt"):
        t, n, r, m, o = c["rows"], c["adapters"], c["rank"], c["n_in"], c["n_out"]
        s.ids = _adapter_ids(c, seed)
        s.x = _rows(seed, 11, t, m, c["pad"])
        s.a = _normal(seed, 12, (n, r, m), m ** -0.5)
        s.b = _normal(seed, 13, (n, o, r), r ** -0.5)
        s.scale = torch.rand((n,), generator=_generator(seed, 14), device=DEV) + 0.5
        if c["kind"] == "adapt":
            s.base = _rows(seed, 15, t, o, c["pad"])
            s.out = torch.empty((t, o), dtype=torch.bfloat16, device=DEV)
        else:
            s.dy, s.dx_base = _rows(seed, 16, t, o, c["pad"]), _rows(seed, 17, t, m, 0)
            s.h = _normal(seed, 18, (t, r), dtype=torch.float32) * (s.ids >= 0)[:, None]       # what a forward pass kept
            s.dx = torch.empty((t, m), dtype=torch.bfloat16, device=DEV)
            s.da, s.db = torch.empty_like(s.a), torch.empty_like(s.b)
        if own:
            from paper_2605_22428_amd import binding as B
            s.adapters = B.Adapters(s.a, s.b, s.scale)
            s.workspace = s.adapters.workspace(t)
        return s
    t, e, k = c["tokens"], c["experts"], c["top_k"]
    s.logits = _normal(seed, 21, (t, e), dtype=torch.float32)
    if c["masked"]:                                   # experts out of service, and (of several) a token whose every expert is
        s.logits[torch.rand((t, e), generator=_generator(seed, 22), device=DEV) < c["masked"]] = -math.inf
        s.logits[t // 2:t // 2 + min(1, t // 2)] = -math.inf
    if c["logits"] == "bf16":
        s.logits = s.logits.bfloat16()
    s.bias = _normal(seed, 23, (e,), 0.1, torch.float32) if c["bias"] else None
    s.ids = torch.empty((t, k), dtype=torch.int32, device=DEV)
    s.weights = torch.empty((t, k), dtype=torch.float32, device=DEV)
    if c["kind"] == "route_backward":
        s.ids = _select(c, s.logits, s.bias)[0]
        s.d_weights = _normal(seed, 24, (t, k), dtype=torch.float32)
        s.d_logits = torch.empty_like(s.logits)
    if c["kind"] == "layer":
        n, h, i = _local(c), c["hidden"], c["inter"]
        s.x = _rows(seed, 31, t, h, 0)
        s.gate_up = _normal(seed, 32, (n, 2, i, h), h ** -0.5)
        s.down = _normal(seed, 33, (n, h, i), i ** -0.5)
        s.gate_up_scale = s.down_scale = None
        if c["weights"] == "fp8":
            (s.gate_up, s.gate_up_scale), (s.down, s.down_scale) = _fp8(s.gate_up), _fp8(s.down)
        s.out = torch.empty((t, h), dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2605_22428_amd import binding as B
        place = _placement(c) if c["kind"] == "layer" else np.zeros(e, dtype=np.int32)
        s.ctx = B.Context(c.get("ranks", 1), e, k, 0, c.get("hidden", 8), B.MW_ROW_BF16, t, 0, place)
        s.gate = B.Gate((B.MW_GATE_SOFTMAX, B.MW_GATE_SOFTMAX_TOPK, B.MW_GATE_SIGMOID_TOPK)[SCORES.index(c["score"])],
                        c["groups"], c["kept"], 2.5)
        if c["kind"] == "layer":
            s.experts = B.Experts(s.gate_up, s.down, s.gate_up_scale, s.down_scale)
            s.workspace = s.ctx.moe_workspace(s.experts, t)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def _select(c, logits, bias):
    """(ids, the scores in 32 bits): the K best of score + bias among the kept groups' experts, ties to the lowest id."""
    l = logits.float()
    l = torch.where(l.isnan(), -math.inf, l).clamp(max=BIG)
    by = (l if bias is None else l + bias).clamp(max=BIG)
    if c["groups"] > 1:
        groups = by.unflatten(1, (c["groups"], -1))
        best = groups.sort(dim=2, descending=True).values[:, :, :2].sum(2)
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        allowed = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        by = torch.where(allowed[:, :, None], groups, -math.inf).flatten(1)
    order = by.sort(dim=1, descending=True, stable=True)
    ids = torch.where(order.values > -math.inf, order.indices, -1)[:, :c["top_k"]].int().contiguous()
    return ids, l


def _chosen(c, l, ids):
    """What each chosen expert weighs before the factor (0 where none was chosen), and whether one was."""
    some = ids >= 0
    lk = torch.where(some, l.gather(1, ids.clamp(min=0).long()), -math.inf)
    if c["score"] == "sigmoid_topk":
        v = torch.where(some, 1 / (1 + torch.exp(-lk)), 0)
        total = v.sum(1, keepdim=True)
    else:
        m = (l if c["score"] == "softmax" else lk).amax(1, keepdim=True).clamp(min=-BIG)
        v = torch.where(some, torch.exp(lk - m), 0)
        total = torch.exp(l - m).sum(1, keepdim=True) if c["score"] == "softmax" else v.sum(1, keepdim=True)
    return torch.where(total > 0, v / total, 0), some


def _plain_route(c, logits, bias):
    ids, l = _select(c, logits, bias)
    return ids, _chosen(c, l, ids)[0] * 2.5


def _plain_route_backward(c, logits, ids, dw):
    l = logits.float()
    l = torch.where(l.isnan(), -math.inf, l).clamp(max=BIG)
    q, some = _chosen(c, l, ids)
    g = torch.where(some, dw, 0)
    mean = (g * q).sum(1, keepdim=True)
    at = torch.where(some, ids, c["experts"]).long()
    wide = torch.zeros((l.shape[0], c["experts"] + 1), device=l.device)
    if c["score"] == "softmax":
        m = l.amax(1, keepdim=True).clamp(min=-BIG)
        p = torch.exp(l - m)
        p = p / p.sum(1, keepdim=True).clamp(min=1e-30)
        d = p * (wide.scatter(1, at, g)[:, :-1] - mean)
    else:
        d = q * (g - mean)
        if c["score"] == "sigmoid_topk":
            d = d / (1 + torch.exp(l.gather(1, ids.clamp(min=0).long())))
        d = wide.scatter(1, at, d)[:, :-1]
    return (2.5 * d).to(logits.dtype)


def _plain_layer(s):
    c = s.case
    ids, w = _plain_route(c, s.logits, s.bias)
    up, down = (s.gate_up.float(), s.down.float()) if s.gate_up_scale is None else (_wide(s.gate_up, s.gate_up_scale), _wide(s.down, s.down_scale))
    x = s.x.float()[None, None]
    y = torch.matmul(x, up.transpose(2, 3))                                                   # [experts][2][tokens][inter]
    y = y[:, 0] / (1 + torch.exp(-y[:, 0])) * y[:, 1]
    mine = ids[None] == torch.arange(_local(c), device=DEV)[:, None, None]
    y = y * (mine * w[None]).sum(2)[:, :, None]
    return torch.matmul(y, down.transpose(1, 2)).sum(0).bfloat16(), ids, w


def _own_adapter(s):
    """[rows][adapters]: the factor of a row's own adapter, 0 elsewhere."""
    return (s.ids[:, None] == torch.arange(s.case["adapters"], device=DEV)) * s.scale


def _plain_adapt(s):
    h = torch.matmul(s.x.float(), s.a.float().flatten(0, 1).t()).unflatten(1, (s.case["adapters"], -1)) * _own_adapter(s)[:, :, None]
    return (s.base.float() + torch.matmul(h.flatten(1), s.b.float().transpose(1, 2).flatten(0, 1))).bfloat16()


def _plain_adapt_backward(s):
    n, mine = s.case["adapters"], _own_adapter(s)[:, :, None]
    x, dy = s.x.float(), s.dy.float()
    dh = torch.matmul(dy, s.b.float().transpose(1, 2).flatten(0, 1).t()).unflatten(1, (n, -1)) * mine
    dx = s.dx_base.float() + torch.matmul(dh.flatten(1), s.a.float().flatten(0, 1))
    da = torch.matmul(dh.flatten(1).t(), x).unflatten(0, (n, -1))
    db = torch.matmul((s.h[:, None, :] * mine).flatten(1).t(), dy).unflatten(0, (n, -1)).transpose(1, 2)
    return dx.bfloat16(), da.bfloat16(), db.bfloat16().contiguous()


def run(state):
    s, c = state, state.case
    kind = c["kind"]
    if kind == "route":
        if not own:
            return _plain_route(c, s.logits, s.bias)
        s.ctx.mw_route(s.gate, s.logits, s.bias, s.ids, s.weights)
        return s.ids, s.weights
    if kind == "route_backward":
        if not own:
            return _plain_route_backward(c, s.logits, s.ids, s.d_weights)
        s.ctx.mw_route_backward(s.gate, s.logits, s.ids, s.d_weights, s.d_logits)
        return s.d_logits
    if kind == "layer":
        if not own:
            return _plain_layer(s)
        s.ctx.mw_moe_layer(s.gate, s.logits, s.bias, s.experts, s.x, s.ids, s.weights, s.out, s.workspace)
        return s.out, s.ids, s.weights
    if kind == "adapt":
        if not own:
            return _plain_adapt(s)
        s.adapters.mw_adapt(s.x, s.ids, s.base, s.out, s.workspace)
        return s.out
    if not own:
        return _plain_adapt_backward(s)
    s.adapters.mw_adapt_backward(s.x, s.ids, s.h, s.dy, s.dx_base, s.dx, s.da, s.db, s.workspace)
    return s.dx, s.da, s.db


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def _exact_gate(c, logits, ids):
    """Weights of the given ids, token by token's rule written over whole arrays of doubles; also what backward needs."""
    l = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=BIG, neginf=-math.inf)
    hit = torch.zeros((l.shape[0], c["experts"] + 1), dtype=torch.bool, device=DEV)
    hit.scatter_(1, torch.where(ids >= 0, ids, c["experts"]).long(), True)
    hit = hit[:, :-1]
    if c["score"] == "sigmoid_topk":
        v = torch.sigmoid(l) * hit
        q = v / v.sum(1, keepdim=True)
    else:
        q = torch.softmax(l if c["score"] == "softmax" else l.masked_fill(~hit, -math.inf), 1)
    return l, hit, torch.nan_to_num(q, nan=0.0)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"].startswith("adapt"):
        per = [(s.ids == a).nonzero().view(-1) for a in range(c["adapters"])]
        scale = s.scale.double()
        if c["kind"] == "adapt":
            out = s.base.double()
            for a, at in enumerate(per):
                out[at] += scale[a] * (s.x[at].double() @ s.a[a].double().t().contiguous()) @ s.b[a].double().t().contiguous()
            return out
        dx, da, db = s.dx_base.double(), s.a.double() * 0, s.b.double() * 0
        for a, at in enumerate(per):
            dy = s.dy[at].double() * scale[a]
            dh = dy @ s.b[a].double()
            dx[at] += dh @ s.a[a].double()
            da[a] = dh.t().contiguous() @ s.x[at].double()
            db[a] = dy.t().contiguous() @ s.h[at].double()
        return dx, da, db
    ids = s.ids if c["kind"] == "route_backward" else _select(c, s.logits, s.bias)[0]           # (decided on 32-bit sums by definition)
    l, hit, q = _exact_gate(c, s.logits, ids)
    safe = ids.clamp(min=0).long()
    if c["kind"] == "route_backward":
        g = torch.zeros_like(l).scatter_add_(1, safe, torch.where(ids >= 0, s.d_weights.double(), 0.0))
        d = 2.5 * q * (g - (g * q).sum(1, keepdim=True))
        if c["score"] == "sigmoid_topk":
            d = d * (1 - torch.sigmoid(l))
        return d if c["score"] == "softmax" else d * hit
    w = torch.where(ids >= 0, 2.5 * q.gather(1, safe), 0.0)
    if c["kind"] == "route":
        return None, w
    out = torch.zeros(s.x.shape, dtype=torch.float64, device=DEV)
    for e in range(_local(c)):
        token, slot = (ids == e).nonzero(as_tuple=True)
        up, down = s.gate_up[e], s.down[e]
        up, down = (up.double(), down.double()) if s.gate_up_scale is None else (
            _wide(up, s.gate_up_scale[e], torch.float64), _wide(down, s.down_scale[e], torch.float64))
        x = s.x[token].double()
        act = torch.nn.functional.silu(x @ up[0].t().contiguous()) * (x @ up[1].t().contiguous())
        out[token] += w[token, slot][:, None] * (act @ down.t().contiguous())
    return out, None, w
