"""Lines across whose pieces need more threads than one launch has, and lines of more than 2^30 steps along: every element, over operands
that repeat themselves."""
import numpy as np
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

PERIOD = 4096


def operands(names, inner):
    r = np.random.default_rng(5)
    # gates of 0.73 at most: after a period nothing is left of the state before it
    return {k: r.uniform(-1, 1, (1, PERIOD, inner)).astype(np.float32) for k in names}


def device(a, periods):
    return torch.from_numpy(a).to("cuda:0").repeat(1, periods, 1)


def compare(got, want, bound, periods, name):
    """The first period, any in the middle, the last one: those of three."""
    got = got.view(periods, -1)
    want, bound = (torch.from_numpy(t.reshape(3, -1)).to("cuda:0") for t in (want, bound))
    for n, k in ((0, 0), (periods - 1, 2)):
        assert bool(((got[n].double() - want[k]).abs() <= bound[k]).all()), (name, n)
    for first in range(1, periods - 1, 1 << 12):
        some = got[first:min(first + (1 << 12), periods - 1)]
        assert bool(((some.double() - want[1]).abs() <= bound[1]).all()), (name, first)


def room(elements):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 4 * elements:
        pytest.skip("not enough memory")


# 64 lanes a wave whatever the lines are: 2^32 threads and more forward, and in launches side by side
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("periods,inner", [((1 << 19) + 1, 2), ((1 << 17) + 1, 3), ((1 << 19) + 1, 1)])
def test_forward(periods, inner, reverse):
    print("case", periods, inner, reverse, flush=True)
    room(5 * periods * PERIOD * inner)
    t = operands("zx", inner)
    h0 = np.full((1, inner), 2.0, np.float32)
    h = znn.recurrence_fwd(device(t["z"], periods), device(t["x"], periods), torch.from_numpy(h0).to("cuda:0"), 1, reverse)
    want, bound = gated.recurrence_fwd(np.tile(t["z"], (1, 3, 1)), np.tile(t["x"], (1, 3, 1)), h0, reverse)
    compare(h, want, bound, periods, "h")
    del h
    torch.cuda.empty_cache()


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("periods,inner", [((1 << 18) + 1, 2), ((1 << 16) + 1, 3), ((1 << 18) + 1, 1)])
def test_backward(periods, inner, reverse):
    print("case", periods, inner, reverse, flush=True)
    room(8 * periods * PERIOD * inner)
    t = operands(["gh", "z", "x", "h"], inner)
    h0 = np.full((1, inner), 2.0, np.float32)
    dev = [device(t[k], periods) for k in ("gh", "z", "x", "h")]
    gz, gx, gh0 = znn.recurrence_bwd(*dev, torch.from_numpy(h0).to("cuda:0"), 1, reverse)
    wants, bounds = gated.recurrence_bwd(*(np.tile(t[k], (1, 3, 1)) for k in ("gh", "z", "x", "h")), h0, reverse)
    compare(gz, wants[0], bounds[0], periods, "gz")
    compare(gx, wants[1], bounds[1], periods, "gx")
    assert (np.abs(gh0.cpu().numpy() - wants[2]) <= bounds[2]).all()
    del dev, gz, gx
    torch.cuda.empty_cache()
