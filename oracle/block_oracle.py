"""Plain numpy definition, in 64 bits, of score routing, the residual norm and microscaled 4-bit floats."""
from __future__ import annotations

import numpy as np

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], np.float64)


# ------------------------------------------------------------------------- microscaled 4-bit floats
def mx_quantize(x):
    """(codes uint8 [..., K/2], scales uint8 [..., K/32])"""
    v = np.asarray(x, np.float64).reshape(*np.shape(x)[:-1], -1, 32)
    big = np.abs(v).max(-1)
    bad = ~np.isfinite(v).all(-1)
    _, e = np.frexp(np.where(bad, 1.0, big))                          # big = m * 2^e, m in [1/2, 1)
    X = np.where(big > 0, np.clip(e - 3, -127, 127), -127)
    m = np.abs(np.where(bad[..., None], 0.0, v)) / np.exp2(X.astype(np.float64))[..., None]
    code = np.zeros(v.shape, np.int64)
    for c in range(1, 8):                                             # up to code c where nearer to it, or half way and c even
        half = (GRID[c - 1] + GRID[c]) / 2
        code = np.where((m > half) | ((m == half) & (c % 2 == 0)), c, code)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(v))
    flat = code.reshape(*np.shape(x)[:-1], -1, 2)
    return (flat[..., 0] | (flat[..., 1] << 4)).astype(np.uint8), np.where(bad, 255, X + 127).astype(np.uint8)


def mx_values(codes, scales):
    codes = np.asarray(codes)
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, 32)
    v = np.where(n >= 8, -1.0, 1.0) * GRID[n & 7]
    s = np.where(scales == 255, np.nan, np.exp2(np.asarray(scales, np.float64) - 127))
    return (v * s[..., None]).reshape(*codes.shape[:-1], -1)


def silu(g):
    return g / (1.0 + np.exp(-g))


def product(w, x, idx, swiglu):
    """w [E, N, K], x [T, K] or [T, k, K], idx [T, k] or None -> [T, k, N (/ 2)]"""
    T = x.shape[0]
    idx = np.zeros((T, 1), np.int64) if idx is None else np.clip(idx, 0, w.shape[0] - 1)
    xs = x if x.ndim == 3 else np.broadcast_to(x[:, None], (T, idx.shape[1], x.shape[1]))
    y = np.empty((T, idx.shape[1], w.shape[1]))
    for e in np.unique(idx):
        at = np.nonzero(idx == e)
        y[at] = xs[at] @ w[e].T
    return silu(y[..., 0::2]) * y[..., 1::2] if swiglu else y


# ----------------------------------------------------------------------------------------- routing
def scores(z, score):
    z = z.astype(np.float64)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-z))
    out = np.empty_like(z)
    for t in range(z.shape[0]):
        real = z[t][~np.isnan(z[t])]
        m = real.max() if len(real) else -np.inf
        with np.errstate(invalid="ignore"):
            p = np.where(z[t] == -np.inf, 0.0, np.where(z[t] == m, 1.0, np.exp(z[t] - m)))
        out[t] = p if p.sum() == 0 else p / p.sum()
    return out


def route_scores(z, k, score, n_group, topk_group, group_score, bias, norm, scale):
    T, E = z.shape
    all_scores = scores(z, score)
    bias = np.zeros(E) if bias is None else bias.astype(np.float64)
    idx, w = np.empty((T, k), np.int64), np.empty((T, k))
    size = E // n_group
    for t in range(T):
        s = all_scores[t]
        c = s + bias
        rank = lambda v: -np.inf if np.isnan(v) else v
        # a NaN comes after minus infinity
        order = lambda items, key: sorted(items, key=lambda i: (np.isnan(key(i)), -rank(key(i)), i))
        def group(g):
            v = sorted((rank(x) for x in c[g * size:(g + 1) * size]), reverse=True)
            return v[0] + v[1] if group_score == "top2" and size > 1 else v[0]
        allowed = set(order(range(n_group), group)[:topk_group])
        best = order([e for e in range(E) if e // size in allowed], lambda e: c[e])[:k]
        idx[t] = best
        wt = s[best]
        if norm:
            wt = np.zeros(k) if wt.sum() == 0 else wt / wt.sum()
        w[t] = wt * scale
    return idx, w


# ------------------------------------------------------------------------------------ residual norm
def residual_norm(res, y, slot_w, post_w, gate, scale, pre_w, eps):
    f = lambda v: None if v is None else np.asarray(v, np.float64)
    res, y, slot_w, post_w, gate, pre_w = map(f, (res, y, slot_w, post_w, gate, pre_w))
    rms = lambda v: v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    h = 0.0 if res is None else res
    if y is not None:
        b = (y * (1.0 if slot_w is None else slot_w[..., None])).sum(1)
        if post_w is not None:
            b = rms(b) * post_w
        h = h + scale * (1.0 if gate is None else gate) * b
    return h, rms(h) * (1.0 if pre_w is None else pre_w)
