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


# tiles and the sums behind them, images and rows; few features over many positions
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", [(5, 7, 60), (70, 21, 301), (3, 18, 9001)])
@pytest.mark.parametrize("fn", ["logistic", "silu", "tanh", "gelu"])
def test_gated_unit(f, fo, n, axis, fn):
    """gy v beyond the range where the slope is 0 or small: du is no infinity, and 0 where the slope is."""
    r = np.random.default_rng(9)
    shut = r.random((fo, n)) < 0.5
    u = np.where(shut, -200.0, {"logistic": -60.0, "silu": -60.0, "tanh": 30.0, "gelu": -11.0}[fn]).astype(np.float32)
    gy, v = (r.normal(size=(fo, n)) * 1e20).astype(np.float32), (r.normal(size=(fo, n)) * 1e20).astype(np.float32)
    x, w = r.normal(size=(f, n)).astype(np.float32), r.normal(size=(2 * fo, f)).astype(np.float32)
    lay = lambda m: dev(m.T if axis else m)  # noqa: E731
    back = lambda t: host(t.t() if axis else t)  # noqa: E731
    both = np.concatenate([u, v])
    gx, gw, gb = znn.gated_bwd(lay(gy), lay(x), dev(w), lay(both), fn, axis)
    wants, bounds = gated.gated_bwd(gy, x, w, both, fn)
    for name, got, want, bound in zip(("gx", "gw", "gb"), (back(gx), host(gw), host(gb)), wants, bounds):
        assert np.abs(want).max() < 1e36 and np.isfinite(got).all(), name
        assert (np.abs(got - want) <= bound + 1e-37).all(), name
