"""Plain 64-bit forms of the feed-forward operators -- TEST INFRASTRUCTURE.

Written from the formulas in numpy, a row or a token at a time where that is
the clearest; it shares no code with the library.  Only tests import it.

  rmsnorm, rmsnorm_bwd    h = x + r, y = h w / sqrt(mean h^2 + eps), and the
                          gradient of sum(dy * y) + sum(dh * h) to h and w
  mx8, mx8_values         the 8-bit form of a row's groups of 32, and its values
  route, route_bwd        scores, choice, weights, lists; the gradient of
                          sum(dweights * weights) to the logits
  fp4_quantize, fp4_values  4-bit codes and scales, and their values
  product, routed         w x, by one matrix or by each slot's expert
"""
from __future__ import annotations

import numpy as np

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rmsnorm(x, w, eps, r=None):
    """(h, rstd, y) in 64 bits."""
    h = x.astype(np.float64) + (0.0 if r is None else r.astype(np.float64))
    with np.errstate(all="ignore"):
        rstd = 1.0 / np.sqrt(np.mean(h * h, axis=-1) + eps)
        return h, rstd, h * rstd[..., None] * w.astype(np.float64)


def rmsnorm_bwd(dy, h, w, rstd, dh=None):
    """(dx, dw) of n = h rstd, y = n w."""
    dy, h, w = dy.astype(np.float64), h.astype(np.float64), w.astype(np.float64)
    n = h * rstd[..., None]
    g = dy * w
    dx = rstd[..., None] * (g - n * np.mean(g * n, axis=-1, keepdims=True))
    return dx + (0.0 if dh is None else dh.astype(np.float64)), (dy * n).sum(axis=0)


def _groups(v):
    """Rows padded with zeros and cut into groups of 32."""
    v = np.pad(v, [(0, 0)] * (v.ndim - 1) + [(0, -v.shape[-1] % 32)])
    return v.reshape(*v.shape[:-1], -1, 32)


def scale_exponents(v, top):
    """For every group of 32, the smallest e with max|v| <= top 2^e (at least -127)."""
    a = np.abs(_groups(v)).max(axis=-1)
    e = np.full(a.shape, -127, dtype=np.int64)
    for i in np.ndindex(a.shape):
        if not np.isfinite(a[i]):
            e[i] = 128  # the byte 255
        elif a[i] > 0:
            k = int(np.floor(np.log2(a[i] / top))) - 2
            while top * 2.0 ** k < a[i]:
                k += 1
            e[i] = max(k, -127)
    return e


def e4m3_values(codes):
    """The values of 8-bit floats: 4 exponent bits of bias 7, 3 mantissa bits."""
    c = codes.astype(np.int64)
    s, e, m = c >> 7, (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1.0 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(s == 1, -v, v)


def scale_values(b):
    return np.where(b == 255, np.nan, 2.0 ** (b.astype(np.float64) - 127.0))


def mx8_values(q, scales):
    """What 8-bit codes and their scale bytes stand for."""
    return e4m3_values(q) * np.repeat(scale_values(scales), 32, axis=-1)[..., : q.shape[-1]]


def scores(l, kind):
    """Scores of one token's logits; one that is not above -inf has none."""
    there = l > -np.inf
    s = np.zeros(l.shape)
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            s[there] = 1.0 / (1.0 + np.exp(-l[there].astype(np.float64)))
    elif there.any():
        v = l[there].astype(np.float64)
        e = np.where(v == v.max(), 1.0, np.exp(np.where(v == v.max(), 0.0, v - v.max())))
        s[there] = e / e.sum()
    return s, there


def route(logits, k, bias=None, score="softmax", groups=1, keep=None, renorm=True, scale=1.0):
    """(ids, weights, offsets, order)."""
    T, E = logits.shape
    keep = groups if keep is None else keep
    ids = np.full((T, k), -1, dtype=np.int32)
    weights = np.zeros((T, k))
    for t in range(T):
        s, there = scores(logits[t], score)
        key = s if bias is None else s + bias.astype(np.float64)
        there = there & (key > -np.inf)
        if groups > 1:
            size, rank = E // groups, []
            for g in range(groups):
                own = sorted((key[e] for e in range(g * size, (g + 1) * size) if there[e]), reverse=True)
                if own:
                    rank.append((-sum(own[:2]), g))
            kept = {g for _, g in sorted(rank)[:keep]}
            there = there & np.array([e // size in kept for e in range(E)])
        chosen = sorted((-key[e], e) for e in range(E) if there[e])[:k]
        for j, (_, e) in enumerate(chosen):
            ids[t, j], weights[t, j] = e, s[e]
        if renorm:
            weights[t] /= weights[t].sum() + 1e-20
    weights *= scale
    return (ids, weights, *lists(ids, E))


def lists(ids, E):
    """(offsets, order) of the pairs by expert."""
    flat = ids.ravel()
    by = [[p for p in range(flat.size) if flat[p] == e] for e in range(E)]
    offsets = np.concatenate([[0], np.cumsum([len(b) for b in by])]).astype(np.int32)
    order = np.full(flat.size, -1, dtype=np.int32)
    order[: offsets[-1]] = [p for b in by for p in b]
    return offsets, order


def route_bwd(dweights, logits, ids, score="softmax", renorm=True, scale=1.0):
    """The gradient of sum(dweights * weights) to the logits, by the chain rule."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        s, _ = scores(logits[t], score)
        on = [(j, e) for j, e in enumerate(ids[t]) if 0 <= e < E]
        total = sum(s[e] for _, e in on) + 1e-20
        dot = sum(dweights[t, j] * s[e] for j, e in on)
        ds = np.zeros(E)
        for j, e in on:
            ds[e] = scale * ((dweights[t, j] - dot / total) / total if renorm else dweights[t, j])
        out[t] = ds * s * (1 - s) if score == "sigmoid" else s * (ds - (ds * s).sum())
    return out


def fp4_values(codes, scales, K):
    """Weights of plain codes [..., ceil(K / 2)] and scale bytes [..., ceil(K / 32)]."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)[..., :K]
    v = np.where(c >= 8, -FP4[c & 7], FP4[c & 7])
    return v * np.repeat(scale_values(scales), 32, axis=-1)[..., :K]


def fp4_quantize(w):
    """(codes, scale bytes) of rows of weights: to nearest, ties to the even code."""
    w = w.astype(np.float64)
    K = w.shape[-1]
    b = scale_exponents(w, 6.0) + 127
    u = w / np.repeat(np.where(b == 255, np.inf, scale_values(np.where(b == 255, 0, b))), 32, axis=-1)[..., :K]
    u = np.where(np.isfinite(u), u, 0.0)
    d = np.abs(np.abs(u)[..., None] - FP4)
    near = d == d.min(axis=-1, keepdims=True)
    c = np.where(near.sum(axis=-1) > 1, (near & (np.arange(8) % 2 == 0)).argmax(axis=-1), near.argmax(axis=-1))
    c = (c | np.where(np.signbit(u), 8, 0)).astype(np.uint8)
    c = np.pad(c, [(0, 0)] * (c.ndim - 1) + [(0, K % 2)])
    return c[..., ::2] | c[..., 1::2] << 4, b.astype(np.uint8)


def product(w, x, skip=False):
    """(w x, |w| |x|) for rows of x: the value and the size of its terms; with `skip` an
    x of 0 adds nothing whatever its weights."""
    x = x.astype(np.float64)
    with np.errstate(all="ignore"):
        if not skip:
            return x @ w.T, np.abs(x) @ np.abs(w).T
        y = np.zeros((x.shape[0], w.shape[0]))
        size = np.zeros_like(y)
        for t in range(x.shape[0]):
            on = np.flatnonzero(x[t] != 0)
            y[t] = (w[:, on] * x[t, on]).sum(axis=1)
            size[t] = np.abs(w[:, on] * x[t, on]).sum(axis=1)
        return y, size


def routed(w, x, ids, skip=False):
    """(values, sizes) [T, k, N] of each slot's expert times its row: x [T, K] or [T, k, K]."""
    T, k = ids.shape
    y, size = np.zeros((2, T, k, w.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= ids[t, j] < w.shape[0]:
                row = x[t] if x.ndim == 2 else x[t, j]
                a, b = product(w[ids[t, j]], row[None], skip)
                y[t, j], size[t, j] = a[0], b[0]
    return y, size
