"""What a decoder runs beside the layer calls, in fp64: rotation by position, the paged cache's
layout, causal attention over a sequence, and the choice of a token from logits; norms of heads, and
vectors held in 8 bits.
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


def head_norm(x, weight, eps):
    """Each head (the last dimension) over the root of its mean square, times a weight."""
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)


def _e4m3_values():
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    return np.where(c & 127 == 127, np.nan, np.where(c > 127, -v, v))


E4M3 = _e4m3_values()


def hold(x, least, most):
    """(numbers, exponents) that stand for vectors x along the last dimension in 8 bits: number d is
    x_d / 2^e rounded to e4m3 (nearest, ties to even, at most 448 in magnitude; NaN where x_d is not
    finite), e = ceil(log2(max |x_d| / 448)) over the finite ones, within [least, most]."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x)
    big = np.where(finite, np.abs(x), 0).max(-1)
    f, e = np.frexp(big)  # big = f 2^e, 1/2 <= f < 1; 448 = 7/8 2^9
    e = np.where(big == 0, least, np.clip(e - 9 + (f > 0.875), least, most))
    v = np.where(finite, x, 0) * 2.0 ** -e[..., None].astype(np.float64)
    step = 2.0 ** (np.maximum(np.frexp(v)[1] - 1, -6) - 3.0)
    v = np.clip(np.rint(v / step) * step, -448, 448)
    return np.where(finite, v, np.nan), e


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
