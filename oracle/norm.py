"""Group norm with an activation and dropout over channels-last tensors, and
the counter-based dropout mask: NumPy float64, from the formulas.

Not in the paper (its networks use batch norm, section 4.2); the unit of a
checkpointed net whose statistics do not couple the batch.
"""
from __future__ import annotations

import math

import numpy as np

_M0, _M1, _W0, _W1, _LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def philox4x32_10(counter, key):
    """Four 32-bit words for a counter of four words and a key of two (Salmon,
    Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011);
    words are integers or arrays of them."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k0, k1 = (int(v) for v in key)
    low = np.uint64(_LOW)
    for _ in range(10):
        a, b = c[0] * np.uint64(_M0), c[2] * np.uint64(_M1)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + _W0) & _LOW, (k1 + _W1) & _LOW
    return c


def dropout_factor(count, p, seed, step, site, first=0):
    """What elements first .. first + count - 1 are multiplied by: 0 or the scale."""
    T = math.floor(65536 * p + 0.5)
    e = np.arange(first, first + count, dtype=np.uint64)
    blk, inv = np.unique(e // np.uint64(8), return_inverse=True)
    w = philox4x32_10([blk, np.full_like(blk, site), np.full_like(blk, step & _LOW), np.full_like(blk, step >> 32)],
                      [seed & _LOW, seed >> 32])
    words = np.stack(w, 1)[inv.reshape(-1), ((e % np.uint64(8)) // np.uint64(2)).astype(int)]
    half = (words >> (np.uint64(16) * (e % np.uint64(2)))) & np.uint64(0xFFFF)
    return np.where(half >= T, 65536 / (65536 - T) if T < 65536 else 0.0, 0.0)


def sigmoid(u):
    return 1.0 / (1.0 + np.exp(-u))


def act(kind, u):
    return {"none": lambda: u, "relu": lambda: np.maximum(u, 0.0), "silu": lambda: u * sigmoid(u)}[kind]()


def act_slope(kind, u):
    if kind == "none":
        return np.ones_like(u)
    if kind == "relu":
        return (u > 0).astype(np.float64)
    q = sigmoid(u)
    return q * (1 + u * (1 - q))


def group_stats(x, groups, eps):
    """mean and 1/std, [n, groups], of x [n, hw, c]."""
    n, hw, c = x.shape
    v = np.asarray(x, np.float64).reshape(n, hw, groups, c // groups)
    mean = v.mean((1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean((1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def _spread(v, c):
    return np.repeat(v, c // v.shape[1], 1)[:, None, :]


def _selected(v, factor):
    """v times the factor, 0 where that is 0 (whatever v is)."""
    if factor is None:
        return v
    f = factor.reshape(v.shape)
    with np.errstate(invalid="ignore"):
        return np.where(f == 0, 0.0, v * f)


def gn_apply(x, mean, rstd, gamma, beta, kind="none", factor=None):
    x = np.asarray(x, np.float64)
    c = x.shape[2]
    u = (x - _spread(mean, c)) * _spread(rstd, c) * gamma + beta
    return _selected(act(kind, u), factor)


def affine_f32(x, mean, rstd, gamma, beta):
    """u = (x - mean) (gamma rstd) + beta with every operation rounded to float32:
    the u whose sign ReLU's forward and backward go by."""
    f = np.float32
    c = x.shape[2]
    t = np.asarray(x, f) - _spread(np.asarray(mean, f), c)
    return t * (np.asarray(gamma, f) * _spread(np.asarray(rstd, f), c)) + np.asarray(beta, f)


def gn_backward(g, x, mean, rstd, gamma, beta, kind="none", factor=None, positive=None):
    """(d, dgamma, dbeta); positive: ReLU's decisions (u > 0), else taken in float64."""
    x = np.asarray(x, np.float64)
    n, hw, c = x.shape
    groups = mean.shape[1]
    xhat = (x - _spread(mean, c)) * _spread(rstd, c)
    du = _selected(np.asarray(g, np.float64), factor)
    if kind == "relu":
        du = np.where(xhat * gamma + beta > 0 if positive is None else positive, du, 0.0)
    else:
        du = du * act_slope(kind, xhat * gamma + beta)
    gd = du * gamma
    mean_of = lambda v: _spread(v.reshape(n, hw, groups, c // groups).mean((1, 3)), c)
    d = _spread(rstd, c) * (gd - mean_of(gd) - xhat * mean_of(gd * xhat))
    return d, (du * xhat).sum((0, 1)), du.sum((0, 1))
