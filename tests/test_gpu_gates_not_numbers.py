"""Gates of a gated unit that are NaN, for every function and by every kernel: y and the gradients say so, but for the rectifier,
which is 0 there with a slope of 0."""
import numpy as np
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

FNS = ["rectify", "logistic", "tanh", "silu", "gelu"]


def rows_of(t, axis):
    return (t if axis == 0 else t.t()).cpu().numpy().astype(np.float64)


# one position, a few, tiles of either kind, shares that are joined, few features over many positions
SHAPES = [(40, 24, 1), (40, 24, 20), (70, 33, 300), (1024, 130, 64), (300, 3001, 1025), (40, 24, 33001), (100, 20, 11003)]


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", SHAPES)
@pytest.mark.parametrize("where", ["bias", "weights"])
def test_a_gate_that_is_no_number(f, fo, n, axis, fn, where):
    print("case", f, fo, n, axis, fn, where, flush=True)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    make = lambda *s: torch.randn(s, generator=gen, device="cuda:0")  # noqa: E731
    x, gy = (make(n, k) if axis else make(k, n) for k in (f, fo))
    w, b, m = make(2 * fo, f) / f ** 0.5, make(2 * fo), fo // 2
    (b if where == "bias" else w)[m] = float("nan")
    y, kept = znn.gated_fwd(x, w, b, fn, axis)
    y, both = rows_of(y, axis), rows_of(kept, axis)
    others = np.arange(fo) != m
    assert np.isnan(both[m]).all() and np.isfinite(np.delete(both, m, 0)).all()
    assert np.isfinite(y[others]).all()
    assert (y[m] == 0).all() if fn == "rectify" else np.isnan(y[m]).all()

    gx, gw, gb = znn.gated_bwd(gy, x, make(2 * fo, f), kept, fn, axis)
    gx, gw, gb = rows_of(gx, axis), gw.cpu().numpy(), gb.cpu().numpy()
    halves = np.isin(np.arange(2 * fo), (m, fo + m))
    assert np.isfinite(gw[~halves]).all() and np.isfinite(gb[~halves]).all()
    if fn == "rectify":
        assert (gb[halves] == 0).all() and (gw[halves] == 0).all() and np.isfinite(gx).all()
    else:
        assert np.isnan(gb[halves]).all() and np.isnan(gw[halves]).all() and np.isnan(gx).all()


@pytest.mark.parametrize("axis", [0, 1])
def test_gelu_beside_its_limits(axis):
    """The largest gates and infinite ones, as before: 0 and the gate itself, with slopes of 0 and 1."""
    u = torch.tensor([np.inf, -np.inf, 3.4e38, -3.4e38, 13.0, -13.0, 0.0], device="cuda:0")
    fo = len(u)
    kept = torch.cat([u, torch.full((fo,), 0.5, device="cuda:0")])
    w, x = torch.zeros(2 * fo, 3, device="cuda:0"), torch.ones(3, device="cuda:0")
    y, both = znn.gated_fwd(x.view(-1, 1) if axis == 0 else x.view(1, -1), w, kept, "gelu", axis)
    assert torch.equal(both.flatten(), kept)
    finite = torch.isfinite(u).cpu().numpy()
    want = np.where(finite, gated.gate_fn(np.where(finite, u.cpu().numpy(), 0), "gelu")[0], np.array([np.inf, 0] + [0] * (fo - 2))) * 0.5
    got = y.flatten().cpu().numpy().astype(np.float64)
    assert got[0] == np.inf and got[1] == 0
    # erfc, the product with the gate and that with 0.5: 16 half-steps as for the functions everywhere
    assert (np.abs(got - want)[finite] <= 16 * gated.HALF * np.abs(want)[finite] + 1e-37).all()
    gy = torch.ones_like(y)
    _, _, gb = znn.gated_bwd(gy, x.view(-1, 1) if axis == 0 else x.view(1, -1), w, both, "gelu", axis)
    assert gb[:4].tolist() == [0.5, 0.0, 0.5, 0.0]
