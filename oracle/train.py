"""Plain 64-bit forms of the operators that train a routed block -- TEST INFRASTRUCTURE.

Written from the formulas in numpy; it shares no code with the library.  Only
tests import it.  Next to a result comes its size: the sum of the magnitudes of
the terms that it adds up, which the errors of sums are proportional to.

  lists                   a router's offsets and order from the slots' experts
  expert_linear           v[p] = w[e] x[p], rectified, or summed under weights
  expert_linear_bwd       the gradient of sum(dy * y) to x, w and the weights
  orthogonalize           X <- a X + (b A + c A^2) X, exactly, or with the
                          products' operands rounded to fp16, or to two such parts
"""
from __future__ import annotations

import numpy as np


def lists(ids, E):
    """(offsets [E + 1], order [T * k]): the pairs by expert, in order; -1 behind the last."""
    flat = np.asarray(ids).ravel()
    order = [p for e in range(E) for p in np.flatnonzero(flat == e)]
    counts = [int((flat == e).sum()) for e in range(E)]
    return (np.concatenate([[0], np.cumsum(counts)]).astype(np.int32),
            np.array(order + [-1] * (flat.size - len(order)), dtype=np.int32))


def _pairs(x, k):
    """x's row for every (token, slot)."""
    x = np.asarray(x, dtype=np.float64)
    return np.repeat(x[:, None], k, axis=1) if x.ndim == 2 else x


def expert_linear(x, w, ids, relu=False, weights=None):
    """(y, size): y [T, k, N], or [T, N] with weights."""
    x, w = _pairs(x, ids.shape[1]), np.asarray(w, dtype=np.float64)
    y, size = np.zeros((*ids.shape, w.shape[1])), np.zeros((*ids.shape, w.shape[1]))
    for t, j in np.ndindex(ids.shape):
        if 0 <= ids[t, j] < len(w):
            y[t, j] = w[ids[t, j]] @ x[t, j]
            size[t, j] = np.abs(w[ids[t, j]]) @ np.abs(x[t, j])
    if relu:
        y = np.where(y < 0, 0.0, y)
    if weights is not None:
        s = np.asarray(weights, dtype=np.float64)[..., None]
        return (s * y).sum(1), (np.abs(s) * size).sum(1)
    return y, size


def expert_linear_bwd(dy, x, w, ids, y=None, weights=None):
    """{name: (gradient, size)} of dx, dw and, with weights, dweights.  y: the rectified output."""
    k, shared = ids.shape[1], np.ndim(x) == 2
    x, w, dy = _pairs(x, k), np.asarray(w, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dx, dxs = np.zeros(x.shape), np.zeros(x.shape)
    dw, dws = np.zeros(w.shape), np.zeros(w.shape)
    ds, dss = np.zeros(ids.shape), np.zeros(ids.shape)
    for t, j in np.ndindex(ids.shape):
        e = ids[t, j]
        if not 0 <= e < len(w):
            continue
        d = dy[t] if weights is not None else dy[t, j]
        if y is not None:
            d = np.where(np.asarray(y)[t, j] > 0, d, 0.0)
        s = 1.0 if weights is None else float(weights[t, j])
        back, size = d @ w[e], np.abs(d) @ np.abs(w[e])
        dx[t, j], dxs[t, j] = s * back, abs(s) * size
        dw[e] += s * np.outer(d, x[t, j])
        dws[e] += abs(s) * np.outer(np.abs(d), np.abs(x[t, j]))
        ds[t, j], dss[t, j] = back @ x[t, j], size @ np.abs(x[t, j])
    if shared:
        dx, dxs = dx.sum(1), dxs.sum(1)
    out = {"dx": (dx, dxs), "dw": (dw, dws)}
    if weights is not None:
        out["dweights"] = (ds, dss)
    return out


def _f16(v):
    return v.astype(np.float16).astype(np.float64)


def _two(v):
    """v as an fp16 value and what that leaves, times 2^11, in fp16."""
    high = _f16(v)
    return high + _f16((v - high) * 2048) / 2048


def orthogonalize(g, coefficients, eps, rounded=False):
    """One matrix, in its own orientation; rounded: the products' operands in fp16 (times 2^6), or, "parts", in two
    such values each, and so the state."""
    x = np.asarray(g, dtype=np.float64)
    with np.errstate(all="ignore"):
        x = x / (np.sqrt((x * x).sum()) + eps)
        r = (lambda v: _two(64 * v) / 64) if rounded == "parts" else (lambda v: _f16(64 * v) / 64) if rounded else (lambda v: v)  # noqa: E731
        for a, b, c in coefficients:
            o = r(x)
            x = o if rounded == "parts" else x
            s = r(o @ o.T if x.shape[0] <= x.shape[1] else o.T @ o)
            p = r(b * s + c * (s @ s))
            x = a * x + (p @ o if x.shape[0] <= x.shape[1] else o @ p)
    return x
