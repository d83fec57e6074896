"""Plain 64-bit reference of the low-rank adapters beside a frozen layer and of
gradient clipping (test infrastructure; shares no code with the GPU path)."""
from __future__ import annotations

import numpy as np


def members(ids, g):
    """Row indices of every adapter 0 .. g - 1 that has rows."""
    ids = np.asarray(ids)
    return {k: np.nonzero(ids == k)[0] for k in range(g) if np.any(ids == k)}


def forward(x, w, bias, down, up, scale, ids, relu=False):
    """(y, t) with t = down x of each row's adapter (zeros without one)."""
    n, r = x.shape[0], down.shape[1]
    t = np.zeros((n, r))
    y = x @ w.T
    if bias is not None:
        y = y + bias
    for k, rows in members(ids, down.shape[0]).items():
        t[rows] = x[rows] @ down[k].T
        y[rows] += scale[k] * (t[rows] @ up[k])
    return (np.maximum(y, 0.0) if relu else y), t


def backward(x, w, down, up, scale, ids, dy, t, relu_input=False):
    """(ddown, dup, dx)."""
    ddown, dup = np.zeros_like(down), np.zeros_like(up)
    dx = dy @ w
    for k, rows in members(ids, down.shape[0]).items():
        dt = scale[k] * (dy[rows] @ up[k].T)
        ddown[k] = dt.T @ x[rows]
        dup[k] = scale[k] * (t[rows].T @ dy[rows])
        dx[rows] += dt @ down[k]
    return ddown, dup, (np.where(x > 0, dx, 0.0) if relu_input else dx)


def clip(grads, max_norm):
    """(norm, coefficient): 1 where the norm is zero or not finite."""
    norm = float(np.sqrt(sum(float(np.sum(np.square(g, dtype=np.float64))) for g in grads)))
    return norm, (min(1.0, max_norm / norm) if 0.0 < norm < np.inf else 1.0)
