"""Pins of the reference that the dropout and layer norm kernels are held to: known answers of the generator, shares of
dropped elements, and the gradients against differences in 64 bits."""
import math

import numpy as np
import pytest

from oracle import norm


@pytest.mark.parametrize("counter,key,answer", [
    # known answers of the generator's authors for ten rounds
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_known_answers(counter, key, answer):
    assert tuple(int(v) for v in norm.philox(counter, key)) == answer


def test_words_are_a_function_of_the_place():
    all_of = norm.words(7, 23, 2 ** 40 + 5, 2 ** 33 + 9, 3)
    assert np.array_equal(all_of[2:5, 8:23], norm.words(3, 15, 2 ** 40 + 5, 9, 3, first_row=2, first_col=8))
    for other in (norm.words(7, 23, 2 ** 40 + 6, 9, 3), norm.words(7, 23, 2 ** 40 + 5, 10, 3), norm.words(7, 23, 2 ** 40 + 5, 9, 4)):
        assert (other == all_of).mean() < 0.02


@pytest.mark.parametrize("p", [0.05, 0.25, 0.5, 0.9])
def test_share_of_kept_elements_and_mean(p):
    f = norm.dropout_factor(211, 1003, p, 77, 1)
    n = f.size
    # a binomial share lies within five deviations but for one draw in a million
    assert abs((f > 0).mean() - (1 - p)) < 5 * math.sqrt(p * (1 - p) / n)
    keep = norm.keep_count(p)               # the whole number nearest to (1 - p) 2^32, whose rounding here is below 2^-20
    assert abs(keep - (1 - p) * 2 ** 32) <= 0.5 + 2 ** -20
    assert f.max() == 2 ** 32 / keep


def test_the_ends_of_the_range():
    assert (norm.dropout_factor(3, 5, 0.0) == 1).all()
    assert (norm.dropout_factor(3, 5, 1.0) == 0).all()


@pytest.mark.parametrize("rows,cols,axis", [(3, 5, 1), (5, 3, 0), (1, 4, 1), (4, 1, 1), (6, 1, 0), (1, 6, 0)])
def test_gradients_against_differences(rows, cols, axis):
    rs = np.random.RandomState(rows * 10 + cols)
    x, gy = rs.randn(rows, cols) + 0.5, rs.randn(rows, cols)
    n = (rows, cols)[axis]
    w, b, eps = 1 + 0.3 * rs.randn(n), rs.randn(n), 1e-3
    value = lambda x, w, b: (norm.layernorm_fwd(x, w, b, eps, axis)[0] * gy).sum()  # noqa: E731
    _, m, s = norm.layernorm_fwd(x, w, b, eps, axis)
    for which, got in enumerate(norm.layernorm_bwd(gy, x, w, m, s, axis)):
        args = [x, w, b]
        for at in np.ndindex(args[which].shape):
            def moved(d):
                a = args[which].copy()
                a[at] += d
                return value(*[a if i == which else v for i, v in enumerate(args)])
            # fourth order in the step: differences of 1e-3 leave 1e-12 h and 1e-13 / 1e-3 by rounding
            d = 1e-3
            slope = (8 * (moved(d) - moved(-d)) - (moved(2 * d) - moved(-2 * d))) / (12 * d)
            scale = max(1.0, float(s.max()) ** 5)       # the fifth derivative grows with 1 / deviation where it is that small
            assert abs(slope - got[at]) < 1e-9 * scale, (which, at)


def test_gradients_of_a_net_with_norms_and_dropout():
    """A round's gradients against differences of its loss, with the round's factors held."""
    from oracle import net as onet
    layers = [("conv", 1, 3, (1, 2, 2)), ("layernorm", 1e-3), ("transfer", "tanh"), ("dropout", 0.4), ("conv", 3, 2, (1, 2, 2)),
              ("layernorm",), ("transfer", "logistic")]
    rs = np.random.RandomState(3)
    x, t = rs.randn(1, 1, 5, 6), rs.rand(2, 1, 3, 4)
    params = [{"w": rs.randn(3, 1, 1, 2, 2)}, {"w": 1 + 0.2 * rs.randn(3), "b": rs.randn(3)}, {"b": rs.randn(3)}, None,
              {"w": rs.randn(2, 3, 1, 2, 2)}, {"w": 1 + 0.2 * rs.randn(2), "b": rs.randn(2)}, {"b": rs.randn(2)}]
    factors = {3: norm.dropout_factor(3, 20, 0.4, 5, 1, 3).reshape(3, 1, 4, 5)}
    assert (factors[3] == 0).any() and (factors[3] > 0).any()
    grads = onet.train_round(layers, params, x, t, 0.0, factors=factors)[3]
    for l, p in enumerate(params):
        for k in p or ():
            for at in np.ndindex(p[k].shape):
                def moved(d):
                    q = [None if v is None else {n: a.copy() for n, a in v.items()} for v in params]
                    q[l][k][at] += d
                    return onet.train_round(layers, q, x, t, 0.0, factors=factors)[0]
                d = 1e-4
                slope = (8 * (moved(d) - moved(-d)) - (moved(2 * d) - moved(-2 * d))) / (12 * d)
                # two maps normalise to +-1 steeply where they are near each other: eps = 1e-5 makes fifth derivatives of 1e7 at worst
                assert abs(slope - grads[l][k][at]) < 1e-6 * max(1.0, abs(grads[l][k][at])), (l, k, at)
