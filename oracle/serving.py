"""What a decoder runs beside the layer calls, in fp64: rotation by position, the paged cache's
layout, causal attention over a sequence, and the choice of a token from logits.
"""
import numpy as np


def rotate(x, positions, freqs, adjacent=False):
    """x [tokens, heads, dim] with its first 2 * len(freqs) elements turned by position * freq."""
    x = np.array(x, np.float64)
    half = len(freqs)
    if not half:
        return x
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if adjacent
            else (slice(0, half), slice(half, 2 * half)))
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a] = xa * c - xb * s
    x[..., b] = xb * c + xa * s
    return x


def key_place(t, d):
    """Indices of element d of the token at place t of a page, behind [page, head]."""
    return t // 16, d // 8, t % 16, d % 8


def value_place(t, d):
    return t // 16, t // 8 % 2, d, t % 8


def attend(q, k, v, positions, scale, window=0):
    """(out, weight) of rows q [n, heads, dim] at `positions` over one sequence's k, v
    [tokens, kv_heads, dim]: softmax(scale q.k) v over the keys each row sees, 0 where it sees
    none, and the same with |v|, the scale of its rounding errors."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    t = np.arange(k.shape[0])
    p = np.asarray(positions)[:, None]
    sees = (t <= p) & ((t > p - window) if window else True)
    out, weight = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(n):
        at = np.flatnonzero(sees[i])
        if not at.size:
            continue
        for h in range(heads):
            kk, vv = k[at, h // group].astype(np.float64), v[at, h // group].astype(np.float64)
            s = kk @ q[i, h].astype(np.float64) * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], weight[i, h] = w @ vv, w @ np.abs(vv)
    return out, weight


def choose(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row of logits: the filters in this order, then the first kept
    index at which the running mass exceeds u times the mass."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    top = z.max()
    if top == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(np.argmax(z)), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        x = (z - top) / temperature
        x = np.where(z == top, 0.0, np.where(np.isnan(x), -np.inf, x))
    w = np.where(z == -np.inf, 0.0, np.exp(x))
    order = np.lexsort((np.arange(z.size), -z))
    if 0 < top_k < z.size:
        order = order[:top_k]
    if top_p < 1:
        mass = w[order]
        keep = np.concatenate([[0.0], np.cumsum(mass)[:-1]]) < top_p * mass.sum()
        keep[0] = True
        order = order[keep]
    order = np.sort(order[~(w[order] < min(min_p, 1.0))])
    up = np.cumsum(w[order])
    u = u if u > 0 else 0.0
    i = int(np.searchsorted(up, u * up[-1], side="right"))
    if i >= up.size or w[order[i]] == 0:  # u at or past 1: the last one with any weight
        i = int(np.flatnonzero(w[order])[-1])
    return int(order[i]), float(w[order[i]] / up[-1])
