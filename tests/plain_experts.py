"""Plain 64-bit forms of the experts' products over dispatched rows, and how far fp32 sums and the roundings between them may be off.

u = 2^-24.  A sum of n products in fp32 is off by at most (n + 16) u of the sum of their sizes, whatever its order.  A rounding to bf16 is off by 2^-8 of the
value, sigmoids and the products around them by 16 u."""
import numpy as np

U = 2.0 ** -24
BF16 = 2.0 ** -8


def sums(n):
    return (n + 16) * U


def sig(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def product(a, b, ea=0.0):
    """(a b^T, its error) for rows a that are off by ea."""
    return a @ b.T, ea @ np.abs(b).T + sums(a.shape[1]) * ((np.abs(a) + ea) @ np.abs(b).T) if np.ndim(ea) else sums(a.shape[1]) * (np.abs(a) @ np.abs(b).T)


def block(x, gate_up, down, w):
    """((y, its error), (g and u [rows][2][inter], their error)) of one expert's rows."""
    (g, eg), (u, eu) = product(x, gate_up[0]), product(x, gate_up[1])
    silu = g * sig(g)
    h = silu * u
    eh = 1.1 * np.abs(u) * eg + np.abs(silu) * eu + 1.1 * eg * eu + 16 * U * np.abs(h)
    eh = eh + BF16 * (np.abs(h) + eh)
    y, ey = product(h, down, eh)
    return (w[:, None] * y, np.abs(w)[:, None] * (ey + 2 * U * np.abs(y))), (np.stack((g, u), 1), np.stack((eg, eu), 1))


def block_backward(x, gate_up, down, w, kept, dy):
    """dx, d_gate_up, d_down, dw of one expert's rows, each with its error."""
    g, u = kept[:, 0], kept[:, 1]
    s = sig(g)
    silu, slope = g * s, s * (1 + g * (1 - s))
    h, w = silu * u, w[:, None]
    da, ea = product(dy, down.T)
    dw, edw = (da * h).sum(1), (ea * np.abs(h)).sum(1) + sums(2 * h.shape[1]) * (np.abs(da * h)).sum(1) + 16 * U * np.abs(da * h).sum(1)

    def rounded(v, e):
        e = e + 16 * U * np.abs(v)
        return v, e + BF16 * (np.abs(v) + e)

    # sig (1 + g (1 - sig)) is made as sig + g sig (1 - sig): off by parts of its terms
    dg, edg = rounded(w * da * u * slope, np.abs(w * u) * (np.abs(slope) * ea + 16 * U * np.abs(da) * (s + np.abs(silu))))
    du, edu = rounded(w * da * silu, np.abs(w * silu) * ea)
    hw, ehw = rounded(w * h, 0.0)
    d, ed = np.concatenate((dg, du), 1), np.concatenate((edg, edu), 1)
    dx, edx = product(d, np.concatenate((gate_up[0], gate_up[1])).T, ed)
    dgu, edgu = product(d.T, x.T, ed.T)
    dd, edd = product(hw.T, dy.T, ehw.T)
    shape = gate_up.shape
    return (dx, edx), (dgu.reshape(shape), edgu.reshape(shape)), (dd.T, edd.T), (dw, edw)


def codes_of(x):
    """(codes, scales in float32) of bf16 rows; halves of 127 x / a are exact in 64 bits, and nothing else comes near one."""
    a = np.abs(x).max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        codes = np.where(a > 0, np.rint(127 * x / a), 0.0)
    return codes, (a[:, 0].astype(np.float32) / np.float32(127)).astype(np.float32)


def bf16(v):
    b = np.asarray(v, dtype=np.float32).view(np.uint32)
    return ((b + 0x7fff + ((b >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)
