"""Plain 64-bit reference of the dense layer, group norm and dropout (test infrastructure;
shares no code with the GPU path)."""
from __future__ import annotations

import math

import numpy as np
from scipy.special import erfc, expit


def act(z, name):
    if name == "relu":
        return np.where(z > 0, z, np.where(z <= 0, 0.0, z))         # NaN stays
    if name == "silu":
        return z * expit(z)
    if name == "gelu":
        return 0.5 * z * erfc(-z / math.sqrt(2.0))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        return expit(z) * (1.0 + z * expit(-z))
    if name == "gelu":
        return 0.5 * erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def dense(x, w, bias=None, residual=None, name="none"):
    """(y, z)."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    y = act(z, name)
    return (y if residual is None else y + residual), z


def dense_back(x, w, dy, pre=None, name="none"):
    """(dx, dw, dbias)."""
    dz = dy if pre is None else np.where(dy == 0, 0.0, dy * slope(pre, name))
    return dz @ w, dz.T @ x, dz.sum(0)


def _spread(v, per):
    return np.repeat(v, per, axis=-1)[:, None, :]


def moments(x, groups, eps):
    """(mean, rstd) of samples x groups; x: samples x positions x channels."""
    n, p, c = x.shape
    v = x.reshape(n, p, groups, c // groups)
    mean = v.mean((1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean((1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def norm(x, groups, eps=1e-5, weight=None, bias=None, name="none"):
    """(y, mean, rstd)."""
    per = x.shape[2] // groups
    mean, rstd = moments(x, groups, eps)
    p = (x - _spread(mean, per)) * _spread(rstd, per)
    if weight is not None:
        p = p * weight
    if bias is not None:
        p = p + bias
    return act(p, name), mean, rstd


def norm_back(x, groups, mean, rstd, dy, weight=None, bias=None, name="none"):
    """(dx, dweight, dbias) with the statistics given."""
    n, pos, c = x.shape
    per = c // groups
    w = np.ones(c) if weight is None else weight
    xh = (x - _spread(mean, per)) * _spread(rstd, per)
    dp = dy * slope(xh * w + (0.0 if bias is None else bias), name)
    dh = dp * w
    group_mean = lambda v: _spread(v.reshape(n, pos, groups, per).mean((1, 3)), per)
    dx = _spread(rstd, per) * (dh - group_mean(dh) - xh * group_mean(dh * xh))
    return dx, (dp * xh).sum((0, 1)), dp.sum((0, 1))


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al., SC'11) in whole numbers: four words of 32 bits."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keep(rows, cols, p, seed, site, step):
    """(rows x cols truth values, scale) of the values of the given row numbers that are kept."""
    t = round(65536 * p)
    keep = np.zeros((len(rows), cols), bool)
    for i, r in enumerate(rows):
        for j in range((cols + 7) // 8):
            w = philox4x32((j, r % 2 ** 32, site, step % 2 ** 32), (seed % 2 ** 32, seed >> 32))
            bits = [v for word in w for v in (word & 0xFFFF, word >> 16)]
            for e in range(min(8, cols - 8 * j)):
                keep[i, 8 * j + e] = bits[e] >= t
    return keep, (65536.0 / (65536 - t) if t < 65536 else 0.0)
