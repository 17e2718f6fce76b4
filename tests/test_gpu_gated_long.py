"""The gated unit over more than 2^31 elements: the last positions, and gradients summed over all of them, against 64 bits."""
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu


def silu(u):
    s, t = torch.sigmoid(u), torch.sigmoid(-u)
    return u * s, s + u * s * t


# by registers and by tiles, rows of features and images; kept values, or those and the operand, have more than 2^31 elements
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", [(32, 17, 70000003), (150, 80, 15000001)])
def test_last_positions_and_sums_over_all(f, fo, n, axis):
    print("case", f, fo, n, axis, flush=True)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    make = lambda k, scale=1.0: torch.randn((n, k) if axis else (k, n), generator=gen, device="cuda:0") * scale  # noqa: E731
    rows = (lambda t, a, b: t[a:b].double()) if axis else (lambda t, a, b: t[:, a:b].t().double())
    x, gy = make(f), make(fo, 1e-2)
    w, b = torch.randn((2 * fo, f), generator=gen, device="cuda:0") / f ** 0.5, torch.randn(2 * fo, generator=gen, device="cuda:0")
    assert max(x.numel(), 2 * fo * n) > 1 << 31
    y, kept = znn.gated_fwd(x, w, b, "silu", axis)
    wd = w.double()
    for first in (0, n // 2, n - 5000):
        some = rows(x, first, first + 5000)
        both, bound = some @ wd.t() + b.double(), gated._sum_bound(f) * gated.HALF * (some.abs() @ wd.abs().t() + b.double().abs())
        assert bool(((rows(kept, first, first + 5000) - both).abs() <= bound).all())
        k = rows(kept, first, first + 5000)
        want = silu(k[:, :fo])[0] * k[:, fo:]
        assert bool(((rows(y, first, first + 5000) - want).abs() <= 20 * gated.HALF * (want.abs() + k[:, fo:].abs() * k[:, :fo].abs().clamp(max=1))).all())
    del y
    gx, gw, gb = znn.gated_bwd(gy, x, w, kept, "silu", axis)
    sums = [torch.zeros(s, dtype=torch.float64, device="cuda:0") for s in ((2 * fo, f), (2 * fo,), (2 * fo, f), (2 * fo,))]
    for first in range(0, n, 1 << 20):
        last = min(n, first + (1 << 20))
        k, g = rows(kept, first, last), rows(gy, first, last)
        a, d = silu(k[:, :fo])
        grad = torch.cat([g * k[:, fo:] * d, g * a], 1)
        size = torch.cat([(g * k[:, fo:]).abs() * (d.abs() + 1), g.abs() * (a.abs() + k[:, :fo].abs().clamp(max=1))], 1)
        some = rows(x, first, last)
        for s, v in zip(sums, (grad.t() @ some, grad.sum(0), size.t() @ some.abs(), size.sum(0))):
            s += v
        if first == 0 or last == n:
            bound = (16 + gated._sum_bound(2 * fo)) * gated.HALF * (size @ wd.abs())
            assert bool(((rows(gx, first, last) - grad @ wd).abs() <= bound).all()), first
    bound = (16 + gated._sum_bound(n)) * gated.HALF
    assert bool(((gw.double() - sums[0]).abs() <= bound * sums[2]).all())
    assert bool(((gb.double() - sums[1]).abs() <= bound * sums[3]).all())


# shares of a sum over more than 17 * 2^16 positions, of 2^24 elements
def test_gradients_of_many_weights_over_many_positions():
    f, fo, n = 2048, 4096, 17 * 65536 + 1
    gen = torch.Generator(device="cuda:0").manual_seed(6)
    x, kept, gy = (torch.randn((n, k), generator=gen, device="cuda:0") for k in (f, 2 * fo, fo))
    w = torch.randn((2 * fo, f), generator=gen, device="cuda:0")
    _, gw, gb = znn.gated_bwd(gy, x, w, kept, "silu", 1, need_gx=False)
    some = torch.tensor([0, 1, 777, fo - 1], device="cuda:0")
    k, v, g = kept[:, some].double(), kept[:, some + fo].double(), gy[:, some].double()
    a, d = silu(k)
    sums, sizes = torch.zeros((8, f), dtype=torch.float64, device="cuda:0"), torch.zeros((8, f), dtype=torch.float64, device="cuda:0")
    grad, size = torch.cat([g * v * d, g * a], 1), torch.cat([(g * v).abs() * (d.abs() + 1), g.abs() * (a.abs() + k.abs().clamp(max=1))], 1)
    for first in range(0, n, 1 << 18):
        part = x[first:first + (1 << 18)].double()
        sums += grad[first:first + (1 << 18)].t() @ part
        sizes += size[first:first + (1 << 18)].t() @ part.abs()
    bound, rows = (16 + gated._sum_bound(n)) * gated.HALF, torch.cat([some, some + fo])
    assert bool(((gw[rows].double() - sums).abs() <= bound * sizes).all())
    assert bool(((gb[rows].double() - grad.sum(0)).abs() <= bound * size.sum(0)).all())
