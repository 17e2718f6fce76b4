"""Norms over long positions: sums of millions of elements against 64 bits.

Tolerances in units of u = 2^-24 and of the terms a result is the sum of.  A sum is made of chains of at most 1024 additions,
whose sums are added in chains again, then by trees: the roundings of n additions of like terms add up to about sqrt(n / 3) u of the
sum (18 u for 1024, and less for the average over many threads), what follows adds one u an operation.  64 u hold for that.  One chain of
2^18 squares of normal values is 955 u low, because terms below half an ulp of the sum are lost: 480 u of 1 / deviation.
"""
import pytest
import torch

from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

TOL = 64 * 2.0 ** -24
EPS = 1e-5
DEV = "cuda:0"


def values(rows, cols, axis, seed, power=1):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    make = lambda *n: torch.randn(*n, generator=gen, device=DEV)  # noqa: E731
    n = (rows, cols)[axis]
    # gradients of one sign, so that what a chain loses is not made up for
    return make(rows, cols) ** power, make(rows, cols) ** 2, 1 + 0.2 * make(n), 0.2 * make(n)


def wide(t, axis):
    """[features, positions] in 64 bits"""
    t = t.double()
    return t if axis == 0 else t.t()


def check_forward(y, stats, x, w, b, axis):
    x, y, w, b, stats = wide(x, axis), wide(y, axis), w.double()[:, None], b.double()[:, None], stats.double()
    m = x.mean(0)
    s = 1 / torch.sqrt(((x - m) ** 2).mean(0) + EPS)
    assert bool(((stats[0] - m).abs() <= TOL * x.abs().mean(0)).all()), ((stats[0] - m) / x.abs().mean(0) / TOL).tolist()
    assert bool(((stats[1] - s).abs() <= TOL * s).all()), ((stats[1] / s - 1) / TOL).tolist()
    h = (x - m) * s
    assert bool(((y - (h * w + b)).abs() <= TOL * ((1 + h.abs()) * w.abs() + b.abs())).all())


def check_backward(got, gy, x, w, stats, axis, gr=None):
    gx, gy, x, w, stats = wide(got[0], axis), wide(gy, axis), wide(x, axis), w.double()[:, None], stats.double()
    h = (x - stats[0]) * stats[1]
    a = gy * w
    want = stats[1] * (a - a.mean(0) - h * (a * h).mean(0))
    terms = stats[1] * (a.abs() + a.abs().mean(0) + h.abs() * (a * h).abs().mean(0))
    if gr is not None:
        want, terms = want + wide(gr, axis), terms + wide(gr, axis).abs()
    assert bool(((gx - want).abs() <= TOL * terms).all()), float(((gx - want).abs() / terms).max() / TOL)
    gw, gb = got[-2].double(), got[-1].double()
    assert bool(((gw - (gy * h).sum(1)).abs() <= TOL * (gy * h).abs().sum(1)).all())
    assert bool(((gb - gy.sum(1)).abs() <= TOL * gy.abs().sum(1)).all())


@pytest.mark.parametrize("rows,cols", [(1 << 20, 1), (1 << 20, 2), ((1 << 20) + 3, 3), ((1 << 22) + 1, 1)])
def test_a_few_columns_of_many_rows(rows, cols):
    x, gy, w, b = values(rows, cols, 0, rows + cols)
    y, stats = znn.layernorm_fwd(x, w, b, EPS, 0)
    check_forward(y, stats, x, w, b, 0)
    check_backward(znn.layernorm_bwd(gy, x, w, stats, 0), gy, x, w, stats, 0)


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_a_join_of_a_few_columns_of_many_rows(p):
    rows, cols = (1 << 20) + 1, 3
    x, gy, w, b = values(rows, cols, 0, 5)
    h, gr, _, _ = values(rows, cols, 0, 6)
    state = znn.random_state(77) if p else None
    r, y, stats = znn.residual_norm_fwd(h, x, w, b, p, state, 4, EPS, 0)
    assert torch.equal(r, x + znn.dropout(h, p, state, 4))
    check_forward(y, stats, r, w, b, 0)
    gx, gh, gw, gb = znn.residual_norm_bwd(gy, gr, r, w, stats, p, state, 4, 0)
    check_backward((gx, gw, gb), gy, r, w, stats, 0, gr)
    assert torch.equal(gh, znn.dropout(gx, p, state, 4))


@pytest.mark.parametrize("rows,cols,axis", [(1, (1 << 25) + 5, 1), (2, (1 << 25) + 5, 1), ((1 << 25) + 5, 1, 0)])
def test_gradients_of_more_parameters_than_one_launch_counts(rows, cols, axis):
    """Sums of 2^25 features' shares by 1024 threads for 16 values would be 2^32 threads: more than a launch may have."""
    x, gy, w, b = values(rows, cols, axis, 9)
    y, stats = znn.layernorm_fwd(x, w, b, EPS, axis)
    check_forward(y, stats, x, w, b, axis)
    check_backward(znn.layernorm_bwd(gy, x, w, stats, axis), gy, x, w, stats, axis)


# cubes of normal values: most terms are small beside the largest, and lost in a long chain
@pytest.mark.parametrize("rows,cols,axis", [(1 << 24, 4, 0), ((1 << 22) + 77, 13, 0), (1, 1 << 26, 1), (2, (1 << 25) + 3, 1)])
def test_positions_that_are_walked(rows, cols, axis):
    x, gy, w, b = values(rows, cols, axis, rows + cols, 3)
    y, stats = znn.layernorm_fwd(x, w, b, EPS, axis)
    check_forward(y, stats, x, w, b, axis)
    check_backward(znn.layernorm_bwd(gy, x, w, stats, axis), gy, x, w, stats, axis)


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("rows,cols,axis", [((1 << 22) + 77, 7, 0), (1, (1 << 24) + 3, 1)])
def test_joins_of_positions_that_are_walked(rows, cols, axis, p):
    x, gy, w, b = values(rows, cols, axis, 7, 3)
    h, gr, _, _ = values(rows, cols, axis, 8)
    state = znn.random_state(78) if p else None
    r, y, stats = znn.residual_norm_fwd(h, x, w, b, p, state, 4, EPS, axis)
    assert torch.equal(r, x + znn.dropout(h, p, state, 4))
    check_forward(y, stats, r, w, b, axis)
    gx, gh, gw, gb = znn.residual_norm_bwd(gy, gr, r, w, stats, p, state, 4, axis)
    check_backward((gx, gw, gb), gy, r, w, stats, axis, gr)
    assert torch.equal(gh, znn.dropout(gx, p, state, 4))


# by tiles, walked, by four lanes, by a wave and by a workgroup a row: arrays whose positions are many times what a chip holds at once
@pytest.mark.parametrize("rows,cols,axis", [(40, 20000003, 0), (129, 16700001, 0), (600, 1300001, 0), (30000001, 16, 1), (16700001, 129, 1), (500000, 2500, 1),
                                            (40000, 20000, 1)])
def test_gradients_of_parameters_over_many_positions(rows, cols, axis):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    n, other = (rows, cols)[axis], 1 - axis
    x, gy = torch.randn(rows, cols, generator=gen, device=DEV), torch.randn(rows, cols, generator=gen, device=DEV)
    gy.mul_(gy).mul_(gy)            # fourth powers: most gradients are small beside the largest
    w, b = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
    _, stats = znn.layernorm_fwd(x, w, b, EPS, axis)
    _, gw, gb = znn.layernorm_bwd(gy, x, w, stats, axis)
    sums = torch.zeros(4, n, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 27) // n)   # so many positions at a time in 64 bits
    for i in range(0, (cols, rows)[axis], step):
        part = (slice(None), slice(i, i + step)) if axis == 0 else slice(i, i + step)
        m, s = stats[:, i:i + step].double().unsqueeze(axis + 1)
        g = gy[part].double()
        h = (x[part].double() - m) * s * g
        sums += torch.stack([h.sum(other), h.abs().sum(other), g.sum(other), g.abs().sum(other)])
    assert bool(((gw - sums[0]).abs() <= TOL * sums[1]).all())
    assert bool(((gb - sums[2]).abs() <= TOL * sums[3]).all())
