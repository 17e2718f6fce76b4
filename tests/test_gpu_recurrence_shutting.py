"""Gates between 87 and 104, whose small factor is below 2^-126 and is a factor all the same."""
import numpy as np
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")


def host(t):
    return t.cpu().numpy().astype(np.float64)


def operands(shape, seed):
    r = np.random.default_rng(seed)
    z = (r.normal(size=shape) * 2 + 1).astype(np.float32)
    x, gh = r.normal(size=shape).astype(np.float32), (1 + r.random(shape)).astype(np.float32)
    return z, x, gh, r.normal(size=(shape[0], shape[2])).astype(np.float32)


# single steps, lines that a lane walks, pieces across and along the fastest extent
SHAPES = [(1, 1, 300), (3, 700, 5), (500, 12, 1), (4, 3000, 1), (140000, 9, 2), (1, 5000, 70)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("reverse", [False, True])
def test_what_is_not_finite_passes_a_gate_that_is_not_quite_shut(shape, reverse):
    z, x, gh, h0 = operands(shape, 3)
    r = np.random.default_rng(4)
    narrow = r.random(shape) < 0.1
    z = np.where(narrow, r.uniform(88, 103.5, shape) * r.choice([-1, 1], shape), z).astype(np.float32)
    x[r.random(shape) < 0.02] = np.inf
    x[r.random(shape) < 0.02] = np.nan
    z[r.random(shape) < 0.1] = -np.inf
    z[r.random(shape) < 0.02] = -104.5
    h0.flat[::3] = np.inf
    h0.flat[1::7] = np.nan
    dz, dx, dg, d0 = dev(z), dev(x), dev(gh), dev(h0)
    h = znn.recurrence_fwd(dz, dx, d0, 1, reverse)
    grads = znn.recurrence_bwd(dg, dz, dx, h, d0, 1, reverse)
    with np.errstate(invalid="ignore"):
        wants = [gated.recurrence_fwd(z, x, h0, reverse)]
        g, b = gated.recurrence_bwd(gh, z, x, host(h), h0, reverse)
    wants += list(zip(g, b))
    for name, got, (want, bound) in zip(("h", "gz", "gx", "gh0"), (h,) + tuple(grads), wants):
        got, want, bound = host(got), want.reshape(tuple(got.shape)), bound.reshape(tuple(got.shape))
        assert np.array_equal(np.isnan(got), np.isnan(want)), name
        same = np.isinf(want)
        assert np.array_equal(got[same], want[same]), name
        finite = np.isfinite(want)
        assert (np.abs(got - want)[finite] <= bound[finite]).all(), name


@pytest.mark.parametrize("inner", [1, 3])
def test_a_large_state_or_operand_times_a_small_gate(inner):
    """One step.  The small factor is rounded to multiples of 2^-149 twice (the exponential, its product with the quotient): it is off by 2^-149 at most,
    and by the half-steps of any gate."""
    z = np.linspace(86, 104.2, 3001, dtype=np.float32)
    z = np.concatenate([z, -z])
    z = np.repeat(z[None, None], inner, 1).transpose(0, 2, 1).reshape(-1, 1, inner) if inner > 1 else z.reshape(-1, 1, 1)
    big = np.float32(1e38)
    state, x = np.where(z < 0, big, np.float32(0)).astype(np.float32), np.where(z > 0, big, np.float32(0)).astype(np.float32)
    h = host(znn.recurrence_fwd(dev(z), dev(x), dev(state[:, 0]), 1))
    want = np.exp(-np.abs(z.astype(np.float64))) / (1 + np.exp(-np.abs(z.astype(np.float64)))) * float(big)
    # the other half of a step has a factor of 1 and an operand of 0
    assert (np.abs(h - want) <= gated.STEP * gated.HALF * want + 2.0 ** -149 * float(big)).all()
    gz, gx, gh0 = (host(t) for t in znn.recurrence_bwd(dev(np.full(z.shape, big)), dev(z), dev(x * 0), dev(h * 0), dev(state[:, 0] * 0), 1))
    small = np.where(z > 0, gx, gh0[:, None])
    assert (np.abs(small - want) <= gated.STEP * gated.HALF * want + 2.0 ** -149 * float(big)).all()


@pytest.mark.parametrize("fn", ["logistic", "silu"])
@pytest.mark.parametrize("axis", [0, 1])
def test_gated_units_far_out(fn, axis):
    u = np.linspace(-103.9, -86, 2000, dtype=np.float32)
    fo = len(u)
    v = np.full(fo, 1e36, np.float32)
    v[::5] = np.inf
    b, w, x = dev(np.concatenate([u, v])), torch.zeros(2 * fo, 2, device="cuda:0"), torch.ones(2, device="cuda:0")
    x = x.view(-1, 1) if axis == 0 else x.view(1, -1)
    y, kept = znn.gated_fwd(x, w, b, fn, axis)
    e = np.exp(u.astype(np.float64))
    a, factor = e / (1 + e), 1.0 if fn == "logistic" else -u.astype(np.float64)
    want = a * v * factor * (1 if fn == "logistic" else -1)
    got = host(y).ravel()
    inf = np.isinf(v)
    assert np.array_equal(got[inf], want[inf])
    # as above, and the product with u: rounded once more where it is subnormal
    bound = (16 * gated.HALF * a * factor + 2.0 ** -149 * (factor + 1)) * v
    assert (np.abs(got - want)[~inf] <= bound[~inf]).all()
