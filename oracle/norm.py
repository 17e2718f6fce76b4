"""Float64 reference of dropout, layer norm and the residual join (TEST INFRASTRUCTURE ONLY).

Arrays are [rows][cols]; axis 0 normalises every column over the rows, axis 1 every row over its columns.  The
generator is Philox4x32 with ten rounds as its authors define it (Salmon, Moraes, Dror, Shaw, "Parallel random
numbers: as easy as 1, 2, 3", SC 2011), written on numpy's 64-bit integers.
"""
from __future__ import annotations

import math

import numpy as np

MULTIPLIERS = (0xD2511F53, 0xCD9E8D57)
INCREMENTS = (0x9E3779B9, 0xBB67AE85)
LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=10):
    """Four words per counter: counter is four arrays (or numbers), key two numbers, all below 2^32."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = np.uint64(MULTIPLIERS[0]) * c[0], np.uint64(MULTIPLIERS[1]) * c[2]
        high = lambda v: v >> np.uint64(32)  # noqa: E731
        c = [high(b) ^ c[1] ^ np.uint64(k[0]), b & LOW, high(a) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(v + d) % 2 ** 32 for v, d in zip(k, INCREMENTS)]
    return c


def words(rows, cols, seed, number, site, first_row=0, first_col=0):
    """The word of every element of rows x cols elements from (first_row, first_col) on; first_col divisible by 4."""
    quads = (cols + 3) // 4
    quad = np.arange(first_col // 4, first_col // 4 + quads, dtype=np.uint64)[None, :]
    row = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    c = philox((quad, row, site, number % 2 ** 32), (seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32))
    return np.stack(np.broadcast_arrays(*c), -1).reshape(rows, 4 * quads)[:, :cols]


def keep_count(p):
    return 2 ** 32 - math.floor(p * 2 ** 32 + 0.5)


def dropout_factor(rows, cols, p, seed=0, number=0, site=0, **first):
    """What every element is multiplied by: 2^32 / K where it is kept, 0 where it is dropped."""
    keep = keep_count(p)
    if keep == 2 ** 32:
        return np.ones((rows, cols))
    kept = words(rows, cols, seed, number, site, **first) < np.uint64(keep)
    return np.where(kept, 2 ** 32 / keep if keep else 0.0, 0.0)


def layernorm_fwd(x, w, b, eps, axis):
    """(y, mean, 1 / deviation)"""
    x = np.asarray(x, dtype=np.float64)
    if axis == 0:
        y, m, s = layernorm_fwd(x.T, w, b, eps, 1)
        return y.T, m, s
    m = x.mean(1)
    s = 1 / np.sqrt(((x - m[:, None]) ** 2).mean(1) + eps)
    return (x - m[:, None]) * s[:, None] * np.asarray(w, np.float64) + np.asarray(b, np.float64), m, s


def layernorm_bwd(gy, x, w, mean, inverse, axis):
    """(gx, gw, gb) with the statistics as they are given"""
    gy, x, w, mean, inverse = (np.asarray(a, dtype=np.float64) for a in (gy, x, w, mean, inverse))
    if axis == 0:
        gx, gw, gb = layernorm_bwd(gy.T, x.T, w, mean, inverse, 1)
        return gx.T, gw, gb
    h = (x - mean[:, None]) * inverse[:, None]
    a = gy * w
    gx = inverse[:, None] * (a - a.mean(1)[:, None] - h * (a * h).mean(1)[:, None])
    return gx, (gy * h).sum(0), gy.sum(0)
