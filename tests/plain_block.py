"""Plain 64-bit forms of the gate, the experts and the adapters, written token by token from their definitions (test oracle)."""
import numpy as np

BIG = np.float32(np.finfo(np.float32).max)
SOFTMAX, SOFTMAX_TOPK, SIGMOID_TOPK = 0, 1, 2


def clean(l):
    """fp32 scores: NaN is -inf, +inf the largest finite value."""
    l = np.asarray(l, dtype=np.float32)
    return np.minimum(np.where(np.isnan(l), -np.inf, l), BIG).astype(np.float32)


def select(l, bias, top_k, n_groups, kept):
    """ids of one token."""
    with np.errstate(over="ignore", invalid="ignore"):
        s = l if bias is None else (l + bias).astype(np.float32)
        s = np.minimum(np.where(np.isnan(s), -np.inf, s), BIG).astype(np.float32)
        if n_groups > 1:
            per = len(s) // n_groups
            score = []
            for g in range(n_groups):
                best = sorted(s[g * per:(g + 1) * per], reverse=True)
                score.append(np.float32(best[0] + best[1]) if per > 1 else best[0])
            order = sorted(range(n_groups), key=lambda g: (-score[g], g))
            for g in order[kept:]:
                s = s.copy()
                s[g * per:(g + 1) * per] = -np.inf
    ids = [e for e in sorted(range(len(s)), key=lambda e: (-s[e], e)) if s[e] > -np.inf][:top_k]
    return ids + [-1] * (top_k - len(ids))


def sig(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.float64(v)))


def shares(l, ids, score):
    """(what each entry of ids weighs before the factor, softmax over all experts or None) of one token, 64 bits."""
    l = l.astype(np.float64)
    q, p = np.zeros(len(ids)), None
    some = [k for k, e in enumerate(ids) if e >= 0]
    if score == SOFTMAX:
        top = max(l.max(), -float(BIG))
        v = np.exp(l - top)
        p = v / v.sum() if v.sum() > 0 else v
        for k in some:
            q[k] = p[ids[k]]
        return q, p
    if score == SOFTMAX_TOPK:
        v = {k: np.exp(l[ids[k]] - max(l[ids[j]] for j in some)) for k in some}
    else:
        v = {k: sig(l[ids[k]]) for k in some}
    total = sum(v.values())
    for k in some:
        q[k] = v[k] / total if total > 0 else 0.0
    return q, p


def route(logits, bias, top_k, score, n_groups=1, kept=1, scale=1.0):
    l = clean(logits)
    ids = np.array([select(row, bias, top_k, n_groups, kept) for row in l], dtype=np.int32).reshape(len(l), top_k)
    w = np.array([shares(row, i, score)[0] * scale for row, i in zip(l, ids)]).reshape(len(l), top_k)
    return ids, w


def route_backward(logits, ids, dw, score, scale=1.0):
    """(gradient, what its rounding errors scale with)."""
    l = clean(logits)
    d, size = np.zeros(l.shape), np.zeros(l.shape)
    for t in range(len(l)):
        at = np.where((ids[t] >= 0) & (ids[t] < l.shape[1]), ids[t], -1)
        q, p = shares(l[t], at, score)
        g = np.where(at >= 0, dw[t].astype(np.float64), 0.0)
        mean, big = (g * q).sum(), (np.abs(g) * q).sum()
        if score == SOFTMAX:
            d[t], size[t] = -scale * p * mean, abs(scale) * p * big
            for k, e in enumerate(at):
                if e >= 0:
                    d[t, e] += scale * p[e] * g[k]
                    size[t, e] += abs(scale * p[e] * g[k])
            continue
        for k, e in enumerate(at):
            if e >= 0:
                f = scale * q[k] * (sig(-l[t, e].astype(np.float64)) if score == SIGMOID_TOPK else 1.0)
                d[t, e] += f * (g[k] - mean)
                size[t, e] += abs(f) * (abs(g[k]) + big)
    return d, size


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1.0 + np.exp(-v))


def layer(x, ids, weights, gate_up, down, slots, gamma):
    """(output, how far fp32 sums may be off) of one rank: x [T][H], gate_up [L][2][I][H], down [L][H][I] as float64; slots: id -> local
    expert or -1.  gamma: relative error of a sum of products against the sum of their sizes."""
    out, off = np.zeros(x.shape), np.zeros(x.shape)
    for t in range(len(x)):
        for e in dict.fromkeys(int(e) for e in ids[t]):
            if e not in slots:
                continue
            w, (wg, wu), wd = sum(float(weights[t, k]) for k in range(ids.shape[1]) if ids[t, k] == e), gate_up[slots[e]], down[slots[e]]
            g, u = wg @ x[t], wu @ x[t]
            dg, du = gamma * (np.abs(wg) @ np.abs(x[t])), gamma * (np.abs(wu) @ np.abs(x[t]))
            act = w * silu(g) * u
            d_act = abs(w) * (1.1 * np.abs(u) * dg + np.abs(silu(g)) * du + 1.1 * dg * du) + 2.0 ** -15 * np.abs(act)
            out[t] += wd @ act
            off[t] += np.abs(wd) @ (d_act + gamma * np.abs(act))
    return out, off


def adapt(x, ids, base, a, b, scale, gamma):
    """(out, h, how far fp32 sums may be off, the same of h); x, base, a, b, scale as float64."""
    h = np.zeros((len(x), a.shape[1]))
    dh, out, off = np.zeros(h.shape), base.copy(), np.zeros(base.shape)
    for t in range(len(x)):
        if 0 <= ids[t] < len(a):
            i = int(ids[t])
            h[t], dh[t] = a[i] @ x[t], gamma * (np.abs(a[i]) @ np.abs(x[t]))
            out[t] += scale[i] * (b[i] @ h[t])
            off[t] = abs(scale[i]) * (np.abs(b[i]) @ (dh[t] + 2.0 ** -15 * np.abs(h[t]) + gamma * np.abs(h[t]))) + gamma * np.abs(base[t])
    return out, h, off, dh


def adapt_backward(x, ids, h, dy, dx_base, a, b, scale, gamma):
    """((dx, its error), (da, its error), (db, its error))."""
    dx, dh, ex, eh = adapt(dy, ids, dx_base, b.transpose(0, 2, 1), a.transpose(0, 2, 1), scale, gamma)
    da, ea, db, eb = (np.zeros(v.shape) for v in (a, a, b, b))
    for i in range(len(a)):
        at = np.nonzero(ids == i)[0]
        da[i], db[i] = scale[i] * dh[at].T @ x[at], scale[i] * dy[at].T @ h[at]
        size = abs(scale[i]) * (2.0 ** -15 + gamma)
        ea[i] = abs(scale[i]) * eh[at].T @ np.abs(x[at]) + size * np.abs(dh[at]).T @ np.abs(x[at])
        eb[i] = size * np.abs(dy[at]).T @ np.abs(h[at])
    return (dx, ex), (da, ea), (db, eb)
