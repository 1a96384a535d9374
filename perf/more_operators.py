"""The products of a rank's experts over the rows that a dispatch brought, and products in 8-bit integers, as timed cases.

listed() names the cases, draw() gives more of the same ranges, prepare() makes what a program holds before the call, run() is one
pass, work() the bytes and operations a pass cannot do without, exact() the results in 64 bits.  Where `own` is true run() makes the
library's calls, else it computes the same in elementary torch operations in 32 bits, rounded once at the end.

Kinds of cases
  ffn           mw_ffn: rows in the order of their experts, as mw_unpack leaves them -> the gated feed-forward block of each row's expert,
                times the row's gate weight; with `kept` the gate and up values that the backward pass reads are returned too
  ffn_backward  mw_ffn_backward: gradients of the rows, of every expert's weights and of the gate weights
  matmul_int8   mw_quantize_rows and mw_matmul_int8: rows to 8-bit codes with a scale each, and their product with matrices of codes with a scale for
                each output channel
  ffn_int8      mw_ffn with experts of 8-bit codes: rows, then the block's inner rows (rounded to bf16) are held in codes with a scale each

Rows behind the last expert's are none of any expert; outputs keep there what they held, zeros here.
"""
import math

import torch

DEV = "cuda:0"
own = False
LARGEST_FLOPS, LARGEST_BYTES = 2.9e12, 3.2e9


def _block(name, kind, rows, experts, hidden, inter, weighted, spare=0, pad=0, kept=False):
    return dict(name=name, kind=kind, rows=rows, experts=experts, hidden=hidden, inter=inter, weighted=weighted, spare=spare, pad=pad, kept=kept)


def _matmul(name, rows, matrices, n_in, n_out, spare=0, pad=0):
    return dict(name=name, kind="matmul_int8", rows=rows, experts=matrices, hidden=n_in, n_out=n_out, spare=spare, pad=pad)


def listed():
    return [
        # token generation on a rank of few tokens: one row reached one of eight experts
        _block("ffn_1row_8e", "ffn", 1, 8, 4096, 1024, True),
        # a decode step of 64 ranks with 64 tokens each, 4 of 256 experts here, top-8: 512 rows, room for some more
        _block("ffn_512row_4e", "ffn", 512, 4, 7168, 2048, True, spare=128),
        # a training step's forward pass on such a rank, keeping what its backward pass reads
        _block("ffn_16384row_4e_kept", "ffn", 16384, 4, 7168, 2048, True, kept=True),
        # odd sizes: experts that got a few rows or none, hidden and inner size no multiples of a tile, rows of wider buffers
        _block("ffn_backward_333row_5e_odd", "ffn_backward", 333, 5, 2880, 1000, True, spare=7, pad=64),
        # a small training step: eight smaller experts, weights applied elsewhere
        _block("ffn_backward_2048row_8e", "ffn_backward", 2048, 8, 4096, 1024, False),
        # the largest: the backward pass of the training step above
        _block("ffn_backward_16384row_4e", "ffn_backward", 16384, 4, 7168, 2048, True),
        # a projection of one token
        _matmul("matmul_int8_1row", 1, 1, 7168, 4096),
        # 16 matrices with a few rows each, odd sizes
        _matmul("matmul_int8_100row_16m_odd", 100, 16, 2880, 1008, spare=28, pad=16),
        # a projection of a prompt batch
        _matmul("matmul_int8_8192row", 8192, 1, 7168, 7168),
        # token generation with quantised experts, two rows an expert
        _block("ffn_int8_16row_8e", "ffn_int8", 16, 8, 4096, 1024, True),
        # the decode step above with quantised experts
        _block("ffn_int8_512row_4e", "ffn_int8", 512, 4, 7168, 2048, True, spare=128),
        # a prompt batch's rows on such a rank
        _block("ffn_int8_16384row_4e", "ffn_int8", 16384, 4, 7168, 2048, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["ffn", "ffn", "ffn_backward", "ffn_backward", "matmul_int8", "ffn_int8"])
    c = dict(kind=kind, rows=_log_int(rng, 1, 16384), experts=rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16, 32]),
             hidden=rng.choice([256, 336, 1024, 2048, 2880, 4096, 7168]), spare=rng.choice([0, 0, 1, 40]), pad=rng.choice([0, 0, 16, 64]))
    if kind == "matmul_int8":
        c["n_out"] = rng.choice([256, 512, 1008, 2048, 2880, 4096, 7168])
        return c
    c.update(inter=rng.choice([256, 512, 768, 1008, 1408, 2048]), weighted=rng.random() < 0.6, kept=kind == "ffn" and rng.random() < 0.5)
    if kind != "ffn_int8" and rng.random() < 0.3:     # bf16 rows of any multiple of 8
        c["hidden"], c["inter"] = c["hidden"] + 8, c["inter"] + 8
    return c


def draw(rng):
    while True:
        c = _draw_once(rng)
        sizes = [v for v in c.values() if not isinstance(v, (str, float))]
        w = work(c)
        held = c["experts"] * 6.0 * c["hidden"] * c.get("inter", c.get("n_out"))
        if 3072 not in sizes and w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES and held <= LARGEST_BYTES:
            return c


def _hit(c):
    """Experts that get rows, on average."""
    return c["experts"] * (1 - (1 - 1 / c["experts"]) ** c["rows"])


def work(case):
    c = case
    t, n, h = float(c["rows"]), c["experts"], c["hidden"]
    if c["kind"] == "matmul_int8":
        o = c["n_out"]
        return {"bytes": 2 * t * h + 2 * t * o + _hit(c) * (h * o + 4.0 * o) + 8.0 * (n + 1), "flops": 2 * t * h * o}
    i = c["inter"]
    matrices, rows = 3.0 * h * i, 2 * t * h
    gate = 4 * t * c["weighted"]
    if c["kind"] == "ffn_backward":
        return {"bytes": 3 * rows + 4 * t * i + 2 * gate + 2 * (_hit(c) + n) * matrices + 8.0 * (n + 1), "flops": 12 * t * h * i}
    held = matrices + 4.0 * (2 * i + h) if c["kind"] == "ffn_int8" else 2 * matrices
    return {"bytes": 2 * rows + (4 * t * i if c["kept"] else 0) + gate + _hit(c) * held + 8.0 * (n + 1), "flops": 6 * t * h * i}


# ---- inputs -----------------------------------------------------------------------------------------
def _generator(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + tag) % (1 << 62))
    return g


def _normal(seed, tag, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_generator(seed, tag), dtype=dtype, device=DEV).mul_(std)


def _codes(w):
    """[..., n_out, n_in] -> codes, and a scale for each output channel."""
    w = w.float()
    scale = w.abs().amax(-1) / 127
    return (w / scale[..., None]).round_().to(torch.int8), scale


def _sizes(c, seed):
    """Rows of every expert: some are more popular than others, some may get none."""
    g = _generator(seed, 3)
    popular = torch.exp(0.5 * torch.randn((c["experts"],), generator=g, device=DEV))
    expert = torch.multinomial(popular, c["rows"], replacement=True, generator=g)
    return torch.bincount(expert, minlength=c["experts"])


class _State:
    pass


def prepare(case, seed):
    c, s = case, _State()
    t, n, h, room = c["rows"], c["experts"], c["hidden"], c["rows"] + c["spare"]
    s.case = c
    sizes = _sizes(c, seed)
    s.offsets = torch.zeros((n + 1,), dtype=torch.int64, device=DEV)
    s.offsets[1:] = sizes.cumsum(0)
    s.sizes = sizes.tolist()
    s.most = max(s.sizes)
    expert = torch.repeat_interleave(torch.arange(n, device=DEV), sizes)
    s.place = expert * s.most + torch.arange(t, device=DEV) - s.offsets[expert]       # of a row among n runs of `most` rows
    s.x = _normal(seed, 11, (room, h + c["pad"]))[:, :h]
    if c["kind"] == "matmul_int8":
        o = c["n_out"]
        s.w, s.w_scale = _codes(_normal(seed, 12, (n, o, h), h ** -0.5))
        s.y = torch.zeros((room, o), dtype=torch.bfloat16, device=DEV)
        if own:
            from paper_2605_22428_amd import binding as B
            s.matrices = B.MatricesInt8(s.w, s.w_scale)
            s.codes = torch.empty((room, h), dtype=torch.int8, device=DEV)
            s.scales = torch.empty((room,), device=DEV)
            s.quantize_rows = B.mw_quantize_rows
        return s
    i = c["inter"]
    s.gate_up, s.down = _normal(seed, 13, (n, 2, i, h), h ** -0.5), _normal(seed, 14, (n, h, i), i ** -0.5)
    s.gate_up_scale = s.down_scale = s.kept = s.row_weights = s.d_row_weights = None
    if c["kind"] == "ffn_int8":
        (s.gate_up, s.gate_up_scale), (s.down, s.down_scale) = _codes(s.gate_up), _codes(s.down)
    if c["weighted"]:
        s.row_weights = torch.rand((room,), generator=_generator(seed, 15), device=DEV)
    if c["kind"] == "ffn_backward":
        s.kept = _normal(seed, 16, (room, 2, i))                                      # what a forward pass kept
        s.dy = _normal(seed, 17, (room, h + c["pad"]))[:, :h]
        s.dx = torch.zeros((room, h), dtype=torch.bfloat16, device=DEV)
        s.d_gate_up, s.d_down = torch.empty_like(s.gate_up), torch.empty_like(s.down)
        if c["weighted"]:
            s.d_row_weights = torch.zeros((room,), device=DEV)
    else:
        s.y = torch.zeros((room, h), dtype=torch.bfloat16, device=DEV)
        if c["kept"]:
            s.kept = torch.zeros((room, 2, i), dtype=torch.bfloat16, device=DEV)
    if own:
        import numpy as np
        from paper_2605_22428_amd import binding as B
        s.ctx = B.Context(1, n, 1, 0, h, B.MW_ROW_BF16, 1, room, np.zeros(n, dtype=np.int32))
        s.experts = B.Experts(s.gate_up, s.down, s.gate_up_scale, s.down_scale)
        s.workspace = s.ctx.ffn_workspace(s.experts, room, backward=c["kind"] == "ffn_backward")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def _spread(s, v):
    """Rows -> [experts][most][width] in 32 bits, zeros where an expert has fewer."""
    wide = torch.zeros((s.case["experts"] * s.most, v.shape[1]), device=DEV)
    wide[s.place] = v[:s.case["rows"]].float()
    return wide.unflatten(0, (s.case["experts"], s.most))


def _gather(s, v, dtype):
    """The way back; zeros behind the last expert's rows."""
    rows = v.flatten(0, 1)[s.place].to(dtype)
    return torch.nn.functional.pad(rows, (0, 0, 0, s.case["spare"]))


def _quantize(v):
    """Rows -> codes and scales: 127 x / largest |x| to the nearest, halves to even (in 64 bits, which keep halves apart)."""
    most = v.abs().amax(-1, keepdim=True)
    return torch.where(most > 0, (127 * v.double() / most).round(), 0), most / 127


def _plain_ffn(s):
    c = s.case
    x = _spread(s, s.x)
    gate, up = torch.matmul(x, s.gate_up[:, 0].float().transpose(1, 2)), torch.matmul(x, s.gate_up[:, 1].float().transpose(1, 2))
    y = torch.matmul(gate / (1 + torch.exp(-gate)) * up, s.down.float().transpose(1, 2))
    if c["weighted"]:
        y = y * _spread(s, s.row_weights[:, None])
    y = _gather(s, y, torch.bfloat16)
    return (y, _gather(s, torch.cat((gate, up), 2), torch.bfloat16).unflatten(1, (2, -1))) if c["kept"] else y


def _plain_ffn_backward(s):
    c = s.case
    x, dy, kept = _spread(s, s.x), _spread(s, s.dy), _spread(s, s.kept.flatten(1))
    gate, up = kept[:, :, :c["inter"]], kept[:, :, c["inter"]:]
    sig = 1 / (1 + torch.exp(-gate))
    act = gate * sig * up
    d_act = torch.matmul(dy, s.down.float())
    d_weights = (d_act * act).sum(2, keepdim=True)
    if c["weighted"]:
        w = _spread(s, s.row_weights[:, None])
        d_act, act = d_act * w, act * w
    d_gate, d_up = d_act * up * sig * (1 + gate * (1 - sig)), d_act * gate * sig
    dx = torch.matmul(d_gate, s.gate_up[:, 0].float()) + torch.matmul(d_up, s.gate_up[:, 1].float())
    d_gate_up = torch.stack((torch.matmul(d_gate.transpose(1, 2), x), torch.matmul(d_up.transpose(1, 2), x)), 1)
    d_down = torch.matmul(dy.transpose(1, 2), act)
    out = (_gather(s, dx, torch.bfloat16), d_gate_up.bfloat16(), d_down.bfloat16())
    return out + (_gather(s, d_weights, torch.float32)[:, 0],) if c["weighted"] else out


def _product(codes, scale, w, w_scale):
    """Sums of code products pass 2^24, where 32 bits stop being exact."""
    return torch.matmul(codes, w.double().transpose(1, 2)).float() * scale * w_scale[:, None, :]


def _plain_matmul_int8(s):
    codes, scale = _quantize(_spread(s, s.x))
    return _gather(s, _product(codes, scale, s.w, s.w_scale), torch.bfloat16)


def _plain_ffn_int8(s):
    codes, scale = _quantize(_spread(s, s.x))
    gate = _product(codes, scale, s.gate_up[:, 0], s.gate_up_scale[:, 0])
    up = _product(codes, scale, s.gate_up[:, 1], s.gate_up_scale[:, 1])
    codes, scale = _quantize((gate / (1 + torch.exp(-gate)) * up).bfloat16().float())
    y = _product(codes, scale, s.down, s.down_scale)
    return _gather(s, y * _spread(s, s.row_weights[:, None]) if s.case["weighted"] else y, torch.bfloat16)


def run(state):
    s, kind = state, state.case["kind"]
    if not own:
        return {"ffn": _plain_ffn, "ffn_backward": _plain_ffn_backward, "matmul_int8": _plain_matmul_int8, "ffn_int8": _plain_ffn_int8}[kind](s)
    if kind == "matmul_int8":
        s.quantize_rows(s.x, s.codes, s.scales)
        s.matrices.mw_matmul_int8(s.codes, s.scales, s.offsets, s.y)
        return s.y
    if kind == "ffn_backward":
        s.ctx.mw_ffn_backward(s.experts, s.x, s.offsets, s.kept, s.dy, s.dx, s.d_gate_up, s.d_down, s.workspace,
                              row_weights=s.row_weights, d_row_weights=s.d_row_weights)
        out = (s.dx, s.d_gate_up, s.d_down)
        return out + (s.d_row_weights,) if s.case["weighted"] else out
    s.ctx.mw_ffn(s.experts, s.x, s.offsets, s.y, s.workspace, row_weights=s.row_weights, kept=s.kept)
    return (s.y, s.kept) if s.case["kept"] else s.y


# ---- the definitions in 64 bits ---------------------------------------------------------------------------
def _exact_codes(v):
    most = v.abs().max(dim=1, keepdim=True).values
    ratio = 127 * v / most.clamp(min=1e-300)
    below = ratio.floor()
    odd = torch.remainder(below, 2) == 1
    return below + ((ratio - below > 0.5) | ((ratio - below == 0.5) & odd)), most / 127


def _exact_product(v, w, w_scale):
    codes, scale = _exact_codes(v)
    return (codes @ w.double().t().contiguous()) * scale * w_scale.double()


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, room, i = c["kind"], c["rows"] + c["spare"], c.get("inter")
    wide = dict(dtype=torch.float64, device=DEV)
    y = torch.zeros((room, c.get("n_out", c["hidden"])), **wide)
    kept = torch.zeros((room, 2, i), **wide) if c.get("kept") else None
    d_weights = torch.zeros((room,), **wide)
    d_gate_up, d_down = (torch.zeros(s.gate_up.shape, **wide), torch.zeros(s.down.shape, **wide)) if kind == "ffn_backward" else (None, None)
    first = 0
    for e, rows in enumerate(s.sizes):
        at = slice(first, first + rows)
        first += rows
        if not rows:
            continue
        x = s.x[at].double()
        w = s.row_weights[at].double()[:, None] if c.get("weighted") else 1.0
        if kind == "matmul_int8":
            y[at] = _exact_product(x, s.w[e], s.w_scale[e])
        elif kind == "ffn_int8":
            act = torch.nn.functional.silu(_exact_product(x, s.gate_up[e, 0], s.gate_up_scale[e, 0]))
            act = (act * _exact_product(x, s.gate_up[e, 1], s.gate_up_scale[e, 1])).bfloat16().double()
            y[at] = w * _exact_product(act, s.down[e], s.down_scale[e])
        elif kind == "ffn":
            gate, up = (x @ m.double().t().contiguous() for m in s.gate_up[e])
            y[at] = w * ((torch.nn.functional.silu(gate) * up) @ s.down[e].double().t().contiguous())
            if kept is not None:
                kept[at, 0], kept[at, 1] = gate, up
        else:
            gate, up, dy = s.kept[at, 0].double(), s.kept[at, 1].double(), s.dy[at].double()
            act, slope = torch.nn.functional.silu(gate), torch.sigmoid(gate) + gate * torch.sigmoid(gate) * torch.sigmoid(-gate)
            d_act = dy @ s.down[e].double()
            d_weights[at] = (d_act * act * up).sum(1)
            d_gate, d_up = w * d_act * up * slope, w * d_act * act
            y[at] = d_gate @ s.gate_up[e, 0].double() + d_up @ s.gate_up[e, 1].double()
            d_gate_up[e, 0], d_gate_up[e, 1] = d_gate.t().contiguous() @ x, d_up.t().contiguous() @ x
            d_down[e] = dy.t().contiguous() @ (w * act * up)
    if kind == "ffn_backward":
        return (y, d_gate_up, d_down, d_weights) if c["weighted"] else (y, d_gate_up, d_down)
    return (y, kept) if kept is not None else y
