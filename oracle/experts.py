"""The operators around a layer of experts and of adapters from their definitions, in 64 bits, in plain numpy on the CPU.

As in operators.py, a function of computed values returns the exact result and how far a 32-bit evaluation may be from it."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126                               # what is below may be a zero in 32 bits


def scores(x, kind):
    """Scores of logits [T, E] in 64 bits, 0 where an expert is out."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return np.where(x >= 0, 1 / (1 + np.exp(-x)), np.exp(x) / (1 + np.exp(x)))
        top = x.max(1, keepdims=True)
        p = np.where(x > -np.inf, np.exp(x - np.where(top > -np.inf, top, 0)), 0)
        return p / np.maximum(p.sum(1, keepdims=True), 1e-300)


def shares(x, kind):
    """Logits of chosen experts [n] -> their shares: the scores divided by their sum, without an underflow."""
    log = -np.logaddexp(0, -x) if kind == "sigmoid" else x
    p = np.exp(log - log.max())
    return p / p.sum()


def spread(x):
    """Each row's largest distance of a logit from the largest one, where that still counts (e^-120 does not), [T, 1]."""
    x = np.asarray(x, np.float64)
    top = np.max(np.where(np.isnan(x), -np.inf, x), 1, keepdims=True)
    with np.errstate(invalid="ignore"):
        d = np.where(np.isfinite(x), top - x, 0)
    return np.minimum(np.nan_to_num(d, nan=0.0, posinf=0.0), 120).max(1, keepdims=True)


def route(x, top, kind="softmax", normalize=False, factor=1.0, bias=None):
    """(ids, weights, bound).  The bound: exp(x - largest) is off by the rounding of the difference (U times it) and 2 U of its own, a sum of
    at most 64 in a lane and then six steps by 70 U, quotient, product and the rest by 8 U: all relative to the weight."""
    x = np.asarray(x, np.float64)
    T, E = x.shape
    s = scores(x, kind)
    with np.errstate(invalid="ignore"):
        c = x.copy() if bias is None else s + np.asarray(bias, np.float64)
    c = np.where(np.isnan(c) | np.isnan(x) | (x == -np.inf), -np.inf, c)
    ids = np.argsort(-c, axis=1, kind="stable")[:, :top].astype(np.int32)
    ids = np.where(np.take_along_axis(c, ids, 1) > -np.inf, ids, -1)
    return ids, *weights(x, ids, kind, normalize, factor)


def weights(x, ids, kind="softmax", normalize=False, factor=1.0):
    """(weights of these ids, bound): see route."""
    x = np.asarray(x, np.float64)
    s, w = scores(x, kind), np.zeros(ids.shape)
    for t in range(len(x)):
        live = ids[t] >= 0
        if live.any():
            w[t, live] = factor * (shares(x[t, ids[t, live]], kind) if normalize else s[t, ids[t, live]])
    return w, np.abs(w) * U * (2 * spread(x) + 90) + TINY


def route_backward(x, ids, dweights, kind="softmax", normalize=False, factor=1.0):
    """(dx, bound): the gradient of sum(weights * dweights) with the ids held.  Every part of it is off by what route says, relative to its size."""
    x = np.asarray(x, np.float64)
    T, E = x.shape
    s = scores(x, kind)
    dx, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        live = [j for j, i in enumerate(ids[t]) if 0 <= i < E and x[t, i] > -np.inf]
        if not live:
            continue
        at = ids[t, live]
        g = np.asarray(dweights, np.float64)[t, live] * factor
        slope = 1 / (1 + np.exp(np.minimum(x[t, at], 700))) if kind == "sigmoid" else 1.0
        if normalize:
            p = shares(x[t, at], kind)
            d, m = p * slope * (g - (g * p).sum()), p * slope * (np.abs(g) + (np.abs(g) * p).sum())
        else:
            d, m = s[t, at] * slope * g, s[t, at] * slope * np.abs(g)
        np.add.at(dx[t], at, d)
        np.add.at(size[t], at, m)
        if kind == "softmax" and not normalize:
            dx[t] -= s[t] * d.sum()
            size[t] += s[t] * m.sum()
    return dx, size * U * (3 * spread(x) + 300) + 4 * TINY


def sort(ids, E):
    """(offsets, index, position) of ids [T, top]."""
    ids = np.asarray(ids)
    T, top = ids.shape
    flat = np.where((ids < 0) | (ids >= E), E, ids).reshape(-1)
    order = np.argsort(flat, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1)[:E])]).astype(np.int32)
    rows = np.arange(T * top)
    index = np.where(rows < offsets[E], order // top, -1).astype(np.int32)
    position = np.empty(T * top, np.int32)
    position[order] = np.where(rows < offsets[E], rows, -1)
    return offsets, index, position.reshape(T, top)


def combine(x, position, weights=None, residual=None):
    """(y, bound): y[t] = residual[t] + sum_j weights[t, j] x[position[t, j]]; every one of at most 65 additions and products rounds by U of what is there."""
    x = np.asarray(x, np.float64)
    T, top = position.shape
    live = (position >= 0) & (position < x.shape[0])
    w = np.where(live, 1.0 if weights is None else np.asarray(weights, np.float64), 0.0)
    y = np.zeros((T, x.shape[1])) if residual is None else np.asarray(residual, np.float64).copy()
    size = np.abs(y)
    for j in range(top):
        rows = np.where(live[:, j, None], x[np.where(live[:, j], position[:, j], 0)] if x.size else 0.0, 0.0)
        y = y + w[:, j, None] * rows
        size = size + np.abs(w[:, j, None] * rows)
    return y, U * (top + 2) * size + TINY


def combine_backward(dy, x, position, weights=None):
    """(dx, its bound, dweights, its bound): a product of two values rounds by U; a dot product of C values is at most C / 16 + 12 additions deep."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    T, top = position.shape
    dx, dw, size = np.zeros_like(x), np.zeros((T, top)), np.zeros((T, top))
    for t in range(T):
        for j in range(top):
            p = position[t, j]
            if 0 <= p < x.shape[0]:
                dx[p] = dy[t] * (1.0 if weights is None else float(weights[t, j]))
                dw[t, j], size[t, j] = (dy[t] * x[p]).sum(), np.abs(dy[t] * x[p]).sum()
    return dx, U * np.abs(dx) + TINY, dw, U * (x.shape[1] / 16 + 12) * size + TINY


# what the second product's left operand is off by, relative to its row's largest value: pairs of bf16, pairs of f16, triples of bf16
TERMS = {("bf16", "bf16"): 2.0 ** -16, ("f16", "f16"): 2.0 ** -21, ("f16", "f32"): 2.0 ** -21, ("bf16", "f32"): 2.0 ** -23}


def adapters(base, x, a, b, groups, scale, x_type, y_type):
    """(y, bound) with the rows in groups[e] changed by adapter e.  The bound: K products exact in 32 bits, summed with U each (2 U where the matrix cores truncate) of
    what they add up to in magnitude; the sum taken apart into 16-bit terms (TERMS, of the row's largest magnitude); the same for R products of up to
    three terms; scaling and the sum with base by 4 U."""
    y, bound = np.array(base, np.float64), U * np.abs(np.asarray(base, np.float64))
    for e, rows in enumerate(groups):
        if len(rows) == 0:
            continue
        xe, ae, be = x[rows].astype(np.float64), a[e].astype(np.float64), b[e].astype(np.float64)
        h, mag = xe @ ae.T, np.abs(xe) @ np.abs(ae).T
        off = 2 * U * (x.shape[1] + 24) * mag + TERMS[x_type, y_type] * np.abs(h).max(1, keepdims=True)
        add = scale[e] * (h @ be.T)
        y[rows] += add
        bound[rows] += abs(scale[e]) * (off @ np.abs(be).T + 2 * U * (3 * a.shape[1] + 4) * ((np.abs(h) + off) @ np.abs(be).T)) + 4 * U * (np.abs(add) + np.abs(y[rows])) + TINY
    return y, bound
