"""Gradients whose factors are large and whose value is not: no partial product leaves the range of fp32."""
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


# single steps, lines that a lane walks, pieces across, along the fastest extent
@pytest.mark.parametrize("shape", [(1, 1, 20000), (20000, 1, 1), (140000, 3, 2), (3, 700, 5), (500, 12, 1), (1, 9000, 1)])
@pytest.mark.parametrize("reverse", [False, True])
def test_recurrence(shape, reverse):
    """Factors f (1 - f) of 2^-66 to 2^-100 beside differences of 2^-60 to 2^90 and gradients of as much: of 2^30 and more where steps follow each
    other, as what passes several shut gates is known to 2^-149 of what it was."""
    r = np.random.default_rng(7)
    z = (r.uniform(46, 69, shape) * r.choice([-1, 1], shape)).astype(np.float32)
    x, h = ((r.normal(size=shape) * 2.0 ** r.uniform(-60, 90, shape)).astype(np.float32) for _ in range(2))
    gh = (r.normal(size=shape) * 2.0 ** r.uniform(-60 if shape[1] == 1 else 30, 90, shape)).astype(np.float32)
    h0 = (r.normal(size=(shape[0], shape[2])) * 2.0 ** r.uniform(-60, 90, (shape[0], shape[2]))).astype(np.float32)
    grads = znn.recurrence_bwd(dev(gh), dev(z), dev(x), dev(h), dev(h0), 1, reverse)
    wants, bounds = gated.recurrence_bwd(gh, z, x, h, h0, reverse)
    assert np.abs(wants[0]).max() < 1e37
    for name, got, want, bound in zip(("gz", "gx", "gh0"), grads, wants, bounds):
        got, want, bound = host(got), want.reshape(tuple(got.shape)), bound.reshape(tuple(got.shape))
        assert np.isfinite(got).all(), name
        assert (np.abs(got - want) <= bound).all(), name
