"""Float64 reference of the gated unit and of the gated recurrence along lines (TEST INFRASTRUCTURE ONLY), with bounds on what
32-bit kernels may be off by.

Features are the rows of matrices [features][positions]; lines are arrays [outer][length][inner].
"""
from __future__ import annotations

import math

import numpy as np

try:
    from scipy.special import erfc as _erfc
except ImportError:                     # pragma: no cover
    _erfc = np.vectorize(math.erfc)

HALF = 2.0 ** -24       # half a step of fp32, relative


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x < 0, e / (1 + e), 1 / (1 + e))


def gate_fn(u, fn):
    """(fn(u), its derivative)"""
    u = np.asarray(u, dtype=np.float64)
    if fn == "rectify":
        return np.where(u > 0, u, 0.0), np.where(u > 0, 1.0, 0.0)
    if fn == "logistic":
        return sigmoid(u), sigmoid(u) * sigmoid(-u)
    if fn == "tanh":
        return np.tanh(u), 4 * sigmoid(2 * u) * sigmoid(-2 * u)
    if fn == "silu":
        return u * sigmoid(u), sigmoid(u) + u * sigmoid(u) * sigmoid(-u)
    phi = 0.5 * _erfc(-u / math.sqrt(2))
    return u * phi, phi + u * np.exp(-u * u / 2) / math.sqrt(2 * math.pi)


def _sum_bound(n):
    """Half-steps, relative to the sum of the terms' sizes, that a sum of n products may be off by: a few for products and what follows,
    and roundings of running sums that point either way."""
    return 8 + 2 * math.sqrt(n)


def gated_fwd(x, w, b, fn):
    """(y, [u; v], bound of y, bound of [u; v])"""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    b = np.zeros(w.shape[0]) if b is None else np.asarray(b, np.float64)
    both = w @ x + b[:, None]
    off = _sum_bound(x.shape[0]) * HALF * (np.abs(w) @ np.abs(x) + np.abs(b)[:, None])
    u, v = np.split(both, 2)
    du, dv = np.split(off, 2)
    a, d = gate_fn(u, fn)
    # the functions are a few roundings off what their argument makes of them; no slope exceeds 1.13
    own = 16 * HALF * (np.abs(a) + np.minimum(np.abs(u), 1))
    return a * v, both, (1.2 * du + own) * (np.abs(v) + dv) + (np.abs(a) + own) * dv + 2 * HALF * np.abs(a * v), off


def gated_bwd(gy, x, w, both, fn):
    """(gx, gw, gb) and their bounds, from [u; v] as they are given"""
    gy, x, w, both = (np.asarray(t, np.float64) for t in (gy, x, w, both))
    u, v = np.split(both, 2)
    a, d = gate_fn(u, fn)
    g = np.concatenate([gy * v * d, gy * a])
    # sizes that bound g and hold what its functions may be off by
    size = np.concatenate([np.abs(gy * v) * (np.abs(d) + 1), np.abs(gy) * (np.abs(a) + np.minimum(np.abs(u), 1))])
    extra = 16
    gx, gw, gb = w.T @ g, g @ x.T, g.sum(1)
    bx = (extra + _sum_bound(w.shape[0])) * HALF * (np.abs(w).T @ size)
    bw = (extra + _sum_bound(x.shape[1])) * HALF * (size @ np.abs(x).T)
    bb = (extra + _sum_bound(x.shape[1])) * HALF * size.sum(1)
    return (gx, gw, gb), (bx, bw, bb)


def _times(a, v):
    with np.errstate(invalid="ignore"):
        return np.where(a == 0, 0.0, a * v)


# Half-steps that one step of a recurrence may add, relative to the sizes it joins: exponential 2, sum 1, quotient 1, product with the
# exponential 1 (a gate: 5, of either kind), product and sum 2; pieces of a line that are joined later round products of gates once more, 2.
STEP = 10


def recurrence_fwd(z, x, h0=None, reverse=False):
    """(h, bound)"""
    z, x = np.asarray(z, np.float64), np.asarray(x, np.float64)
    f, k = sigmoid(z), sigmoid(-z)
    # gates that fp32 cannot tell from 0
    f, k = np.where(f < 2.0 ** -150, 0, f), np.where(k < 2.0 ** -150, 0, k)
    h, bound = np.empty_like(x), np.empty_like(x)
    state = np.zeros_like(x[:, 0]) if h0 is None else np.asarray(h0, np.float64).reshape(x[:, 0].shape)
    size, off = np.abs(state), np.zeros_like(state)
    order = range(x.shape[1] - 1, -1, -1) if reverse else range(x.shape[1])
    for t in order:
        joined = _times(f[:, t], size) + _times(k[:, t], np.abs(x[:, t]))
        off = _times(f[:, t], off) + STEP * HALF * joined
        size = joined
        state = _times(f[:, t], state) + _times(k[:, t], x[:, t])
        h[:, t], bound[:, t] = state, off
    return h, bound + 1e-37


def recurrence_bwd(gh, z, x, h, h0=None, reverse=False):
    """(gz, gx, gh0) and their bounds, with h as it is given"""
    gh, z, x, h = (np.asarray(t, np.float64) for t in (gh, z, x, h))
    f, k = sigmoid(z), sigmoid(-z)
    f, k = np.where(f < 2.0 ** -150, 0, f), np.where(k < 2.0 ** -150, 0, k)
    first = np.zeros_like(h[:, :1]) if h0 is None else np.asarray(h0, np.float64).reshape(h[:, :1].shape)
    before = np.concatenate([h[:, 1:], first], 1) if reverse else np.concatenate([first, h[:, :-1]], 1)
    out = [np.empty_like(x) for _ in range(4)]
    q, size, off = (np.zeros_like(x[:, 0]) for _ in range(3))
    order = range(x.shape[1]) if reverse else range(x.shape[1] - 1, -1, -1)
    for t in order:
        g, size = gh[:, t] + q, np.abs(gh[:, t]) + size
        off = off + HALF * size
        fk = f[:, t] * k[:, t]
        span = np.abs(before[:, t]) + np.abs(x[:, t])
        out[0][:, t], out[1][:, t] = _times(fk, g * (before[:, t] - x[:, t])), _times(k[:, t], g)
        out[2][:, t] = _times(fk, (off + 2 * STEP * HALF * size) * span)
        out[3][:, t] = _times(k[:, t], off + STEP * HALF * size)
        q, size = _times(f[:, t], g), _times(f[:, t], size)
        off = _times(f[:, t], off) + STEP * HALF * size
    shape = h[:, 0].shape
    return (out[0], out[1], q.reshape(shape)), (out[2] + 1e-37, out[3] + 1e-37, off.reshape(shape) + 1e-37)
