"""The reference of the gated unit and the gated recurrence: against loops over scalars and against differences."""
import math

import numpy as np
import pytest

from oracle import gated

FNS = ["rectify", "logistic", "tanh", "silu", "gelu"]
RNG = np.random.default_rng


def scalar_fn(u, fn):
    return {"rectify": max(u, 0.0), "logistic": 1 / (1 + math.exp(-u)), "tanh": math.tanh(u), "silu": u / (1 + math.exp(-u)),
            "gelu": u * (1 + math.erf(u / math.sqrt(2))) / 2}[fn]


@pytest.mark.parametrize("fn", FNS)
def test_functions(fn):
    u = np.array([-3.0, -0.7, 0.2, 1.0, 4.0])
    a, d = gated.gate_fn(u, fn)
    e = 1e-6
    for i, v in enumerate(u):
        assert abs(a[i] - scalar_fn(v, fn)) < 1e-14
        assert abs(d[i] - (scalar_fn(v + e, fn) - scalar_fn(v - e, fn)) / (2 * e)) < 1e-9


@pytest.mark.parametrize("fn", FNS)
def test_gated_unit(fn):
    r = RNG(3)
    f, fo, n = 4, 3, 5
    x, w, b, gy = r.normal(size=(f, n)), r.normal(size=(2 * fo, f)), r.normal(size=2 * fo), r.normal(size=(fo, n))
    y, both, _, _ = gated.gated_fwd(x, w, b, fn)
    for j in range(fo):
        for p in range(n):
            u = b[j] + sum(w[j, i] * x[i, p] for i in range(f))
            v = b[fo + j] + sum(w[fo + j, i] * x[i, p] for i in range(f))
            assert abs(both[j, p] - u) < 1e-13 and abs(both[fo + j, p] - v) < 1e-13 and abs(y[j, p] - scalar_fn(u, fn) * v) < 1e-12
    grads, _ = gated.gated_bwd(gy, x, w, both, fn)
    e = 1e-6
    for t, g in zip((x, w, b), grads):
        for at in np.ndindex(t.shape):
            old, got = t[at], []
            for v in (old + e, old - e):
                t[at] = v
                got.append((gated.gated_fwd(x, w, b, fn)[0] * gy).sum())
            t[at] = old
            assert abs(g[at] - (got[0] - got[1]) / (2 * e)) < 1e-7


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("state", [False, True])
def test_recurrence(reverse, state):
    r = RNG(5)
    shape = (2, 6, 3)
    z, x, gh = r.normal(size=shape), r.normal(size=shape), r.normal(size=shape)
    h0 = r.normal(size=(2, 3)) if state else None
    h, _ = gated.recurrence_fwd(z, x, h0, reverse)
    for o in range(2):
        for i in range(3):
            s = h0[o, i] if state else 0.0
            for t in (range(5, -1, -1) if reverse else range(6)):
                f = 1 / (1 + math.exp(-z[o, t, i]))
                s = f * s + (1 - f) * x[o, t, i]
                assert abs(h[o, t, i] - s) < 1e-14
    grads, _ = gated.recurrence_bwd(gh, z, x, h, h0, reverse)
    e = 1e-6
    for t, g in zip((z, x, h0), grads):
        for at in np.ndindex(t.shape) if t is not None else ():
            old, got = t[at], []
            for v in (old + e, old - e):
                t[at] = v
                got.append((gated.recurrence_fwd(z, x, h0, reverse)[0] * gh).sum())
            t[at] = old
            assert abs(g[at] - (got[0] - got[1]) / (2 * e)) < 1e-8


def test_shut_and_open_gates():
    z, x = np.zeros((1, 4, 1)), np.array([1.0, 2.0, np.nan, 4.0]).reshape(1, 4, 1)
    z[0, 1], z[0, 2] = -np.inf, np.inf
    h, _ = gated.recurrence_fwd(z, x, np.array([[np.nan]]))
    assert np.isnan(h[0, 0, 0]) and h[0, 1:, 0].tolist() == [2.0, 2.0, 3.0]
    (gz, gx, gh0), _ = gated.recurrence_bwd(np.ones((1, 4, 1)), z, x, h, np.array([[np.nan]]))
    assert gz[0, 1:, 0].tolist() == [0.0, 0.0, 1.5 * 1 * 0.25 * 0 + (2.0 - 4.0) * 0.25] and gh0[0, 0] == 0.5
    assert gx[0, :, 0].tolist() == [0.5, 2.5, 0.0, 0.5]
