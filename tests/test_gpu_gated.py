"""The gated unit, forward and backward, against the reference in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

FNS = ["rectify", "logistic", "tanh", "silu", "gelu"]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")


def host(t):
    return t.cpu().numpy().astype(np.float64)


def operands(f, fo, n, seed):
    r = np.random.default_rng(seed)
    one = lambda *s: r.normal(size=s).astype(np.float32)  # noqa: E731
    return one(f, n), one(2 * fo, f) / np.float32(np.sqrt(f)), one(2 * fo), one(fo, n) * np.float32(0.01)


def lay(m, axis):
    return np.ascontiguousarray(m.T if axis else m)


def compare(got, want, bound, name):
    assert got.shape == want.shape, name
    off = np.abs(got - want) / (bound + 1e-37)
    assert np.isfinite(got).all() and off.max() <= 1, (name, off.max())


def check(f, fo, n, axis, fn, seed=3, bias=True, kept=True):
    x, w, b, gy = operands(f, fo, n, seed)
    dx, dw, db, dg = dev(lay(x, axis)), dev(w), dev(b) if bias else None, dev(lay(gy, axis))
    y, both = znn.gated_fwd(dx, dw, db, fn, axis, kept)
    want, wboth, bound, bboth = gated.gated_fwd(x, w, b if bias else None, fn)
    compare(lay(host(y), axis), want, bound, "y")
    if not kept:
        assert both is None
        return
    compare(lay(host(both), axis), wboth, bboth, "kept")
    plain, none = znn.gated_fwd(dx, dw, db, fn, axis, False)
    assert none is None and torch.equal(plain, y)
    grads = znn.gated_bwd(dg, dx, dw, both, fn, axis, bias)
    wants, bounds = gated.gated_bwd(gy, x, w, lay(host(both), axis), fn)
    for name, g, v, e in zip(("gx", "gw", "gb"), grads, wants, bounds):
        if g is not None:
            compare(lay(host(g), axis) if name == "gx" else host(g), v, e, name)
    assert (grads[2] is None) == (not bias)


# single features and positions, one position of many features, few positions, odd numbers around the extents of tiles, many positions of few maps
SHAPES = [(1, 1, 1), (5, 3, 1), (1024, 500, 1), (1001, 77, 1), (130, 40, 2), (257, 33, 3), (64, 65, 4), (100, 31, 5), (515, 70, 8), (48, 64, 9), (33, 20, 17), (1023, 9, 7), (270, 66, 32),
          (259, 5, 33),
          (70, 50, 31), (16, 16, 16), (31, 33, 63), (32, 32, 64), (33, 31, 65), (40, 80, 1728), (127, 129, 130), (128, 128, 128), (129, 127, 257),
          (3, 2, 4099), (2, 5, 10007), (120, 240, 1000), (17, 9, 20011), (300, 5, 777), (5, 300, 776), (260, 515, 300), (1, 64, 515), (64, 1, 515)]


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", SHAPES)
def test_shapes(f, fo, n, axis):
    fn = FNS[(f + fo + n) % 5]
    print("case", f, fo, n, axis, fn, flush=True)
    check(f, fo, n, axis, fn)


# enough tiles for the bf16 matrix cores, in one or all of the products: one step of k and less, whole steps, steps cut short, ragged tiles
LARGE = [(130, 70, 40001), (20, 200, 40000), (32, 64, 70016), (33, 130, 33000), (64, 65, 66000), (95, 96, 45001), (1500, 2800, 300), (1024, 2816, 64),
         (300, 3001, 1025), (1281, 1792, 1100), (127, 33, 9001), (128, 260, 9003), (50, 17, 30001), (81, 16, 13009), (16, 15, 66001), (3, 2, 350003)]


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", LARGE)
def test_large_shapes(f, fo, n, axis):
    fn = FNS[(f + fo + n) % 5]
    print("case", f, fo, n, axis, fn, flush=True)
    check(f, fo, n, axis, fn)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("f,fo,n", [(24, 40, 200), (96, 30, 1), (65, 129, 700)])
def test_functions(f, fo, n, axis, fn):
    check(f, fo, n, axis, fn, 5)
    check(f, fo, n, axis, fn, 7, bias=False)
    check(f, fo, n, axis, fn, 9, kept=False)


@pytest.mark.parametrize("axis", [0, 1])
def test_long_sums(axis):
    """Over 5000 features, and over 300000 positions."""
    check(5003, 33, 70, axis, "silu", 11)
    check(12, 9, 300007, axis, "gelu", 13)


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("n", [1, 300])
def test_gates_far_out_and_not_finite(fn, axis, n):
    """Gates at +-1e-30, +-20, +-100, +-3e38 and at infinity, by their biases alone; factors beside them finite."""
    f = 40
    gates = np.array([0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 100.0, -100.0, 3e38, -3e38, np.inf, -np.inf], np.float32)
    fo = len(gates)
    x, _, _, gy = operands(f, fo, n, 15)
    w = np.zeros((2 * fo, f), np.float32)
    b = np.concatenate([gates, np.full(fo, 0.5, np.float32)])
    y, both = znn.gated_fwd(dev(lay(x, axis)), dev(w), dev(b), fn, axis)
    got = lay(host(both), axis)
    assert np.array_equal(got, np.broadcast_to(b.astype(np.float64)[:, None], got.shape))
    a = {"rectify": np.maximum(gates, 0.0), "logistic": gated.sigmoid(gates.astype(np.float64)), "tanh": np.tanh(gates.astype(np.float64))}.get(fn)
    if a is None:
        a = np.where(np.isinf(gates), np.maximum(gates, 0.0), gated.gate_fn(np.where(np.isinf(gates), 0, gates), fn)[0])
    want = np.broadcast_to((a * 0.5)[:, None], (fo, n))
    out = lay(host(y), axis)
    finite = np.isfinite(want)
    assert np.array_equal(out[~finite], want[~finite])
    assert np.all(np.abs(out - want)[finite] <= 32 * gated.HALF * np.minimum(np.abs(want), 1e38)[finite] + 1e-37)
    gx, gw, gb = znn.gated_bwd(dev(lay(gy, axis)), dev(lay(x, axis)), dev(w), both, fn, axis)
    slopes = {"rectify": (gates > 0) * 1.0, "logistic": gated.gate_fn(gates, "logistic")[1], "tanh": gated.gate_fn(gates, "tanh")[1]}.get(fn)
    if slopes is None:
        slopes = np.where(np.abs(gates) > 1e30, (gates > 0) * 1.0, gated.gate_fn(np.where(np.abs(gates) > 1e30, 0, gates), fn)[1])
    size = np.abs(gy).sum(1) * 0.5
    assert np.all(np.abs(host(gb)[:fo] - gy.astype(np.float64).sum(1) * 0.5 * slopes) <= (32 + 2 * np.sqrt(n)) * gated.HALF * size * (np.abs(slopes) + 1))
    if fn in ("logistic", "tanh"):      # else a factor of the zeros in w is infinite
        assert torch.equal(gx, torch.zeros_like(gx))


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", [(40, 30, 1), (40, 30, 200), (200, 140, 500), (70, 66, 66001), (140, 66, 66001)])
def test_operands_that_are_not_finite_or_at_the_ends_of_the_range(f, fo, n, axis):
    """An infinity or NaN reaches what it is a term of, and nothing else; sums of the largest and smallest numbers are those of fp32."""
    x, w, b, gy = operands(f, fo, n, 17)
    clean, _ = znn.gated_fwd(dev(lay(x, axis)), dev(w), dev(b), "logistic", axis)
    clean = lay(host(clean), axis)
    for bad in (np.inf, np.nan):
        p = n // 2
        x2 = x.copy()
        x2[3, p] = bad
        out = lay(host(znn.gated_fwd(dev(lay(x2, axis)), dev(w), dev(b), "logistic", axis)[0]), axis)
        others = np.arange(n) != p
        assert np.array_equal(out[:, others], clean[:, others])
        with np.errstate(invalid="ignore"):
            both = w.astype(np.float64) @ x2[:, p].astype(np.float64) + b
            want = gated.sigmoid(both[:fo]) * both[fo:]
        assert np.array_equal(np.isnan(out[:, p]), np.isnan(want))
        assert np.array_equal(out[~np.isnan(want) & np.isinf(want), p], want[~np.isnan(want) & np.isinf(want)])
        w2 = w.copy()
        w2[fo + 2, 1] = bad
        out = lay(host(znn.gated_fwd(dev(lay(x, axis)), dev(w2), dev(b), "logistic", axis)[0]), axis)
        rows = np.arange(fo) != 2
        assert np.array_equal(out[rows], clean[rows]) and not np.isfinite(out[2]).any()
    for scale in (1e37, 1e-37):
        xs = x * np.float32(scale)
        _, both = znn.gated_fwd(dev(lay(xs, axis)), dev(w), None, "rectify", axis)
        want, bound = w.astype(np.float64) @ xs, (8 + 2 * np.sqrt(f)) * gated.HALF * (np.abs(w).astype(np.float64) @ np.abs(xs))
        # subnormal terms are rounded to multiples of 2^-149
        assert np.all(np.abs(lay(host(both), axis) - want) <= bound + f * 2.0 ** -149)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", [(33, 21, 5), (40, 30, 200), (70, 66, 33001), (140, 66, 66001), (1281, 1793, 130)])
def test_gradients_of_operands_that_are_not_finite(f, fo, n, axis):
    """An infinity or NaN in one operand reaches the gradients whose sums it is a term of, and no others."""
    x, w, b, gy = operands(f, fo, n, 21)
    _, both, _, _ = gated.gated_fwd(x, w, b, "silu")
    both = both.astype(np.float32)

    def grads(x, w, both, gy):
        got = znn.gated_bwd(dev(lay(gy, axis)), dev(lay(x, axis)), dev(w), dev(lay(both, axis)), "silu", axis)
        return lay(host(got[0]), axis), host(got[1]), host(got[2])

    clean = grads(x, w, both, gy)
    p, m = n // 2, fo // 2
    for bad in (np.inf, np.nan, 3e38):
        g2 = gy.copy()
        g2[m, p] = bad
        gx, gw, gb = grads(x, w, both, g2)
        others = np.arange(n) != p
        assert np.array_equal(gx[:, others], clean[0][:, others])
        rows = np.ones(2 * fo, bool)
        rows[[m, fo + m]] = False
        assert np.array_equal(gw[rows], clean[1][rows]) and np.array_equal(gb[rows], clean[2][rows])
        with np.errstate(invalid="ignore", over="ignore"):
            wants, _ = gated.gated_bwd(g2, x, w, both, "silu")
            for got, want in zip((gx[:, p], gw[[m, fo + m]], gb[[m, fo + m]]), (wants[0][:, p], wants[1][[m, fo + m]], wants[2][[m, fo + m]])):
                want = want.astype(np.float32)
                assert np.array_equal(np.isnan(got), np.isnan(want))
                same = np.isinf(want)
                assert np.array_equal(got[same], want[same])
        x2 = x.copy()
        x2[f // 3, p] = bad
        gx, gw, gb = grads(x2, w, both, gy)
        columns = np.arange(f) != f // 3
        assert np.array_equal(gx, clean[0]) and np.array_equal(gb, clean[2]) and np.array_equal(gw[:, columns], clean[1][:, columns])
        if not np.isfinite(bad):
            assert not np.isfinite(gw[:, f // 3]).any()


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("f,fo,n", [(33, 21, 1), (40, 24, 6), (33, 21, 150), (64, 64, 256), (130, 70, 301), (130, 130, 33001), (1281, 1793, 130), (45, 70, 33001), (100, 20, 11003)])
def test_arrays_on_no_boundary_and_nothing_beside_them(f, fo, n, axis):
    x, w, b, gy = operands(f, fo, n, 19)
    base = [dev(lay(x, axis)), dev(w), dev(b), dev(lay(gy, axis))]
    y, both = znn.gated_fwd(base[0], base[1], base[2], "silu", axis)
    grads = znn.gated_bwd(base[3], base[0], base[1], both, "silu", axis)

    def place(a, first):
        t = torch.full((a.numel() + 8,), 7.5, device="cuda:0")
        t[first:first + a.numel()] = a.reshape(-1)
        return t, t[first:first + a.numel()].view(a.shape)

    L = znn.lib()
    for first in (0, 1, 2, 3):
        (_, px), (_, pw), (_, pb), (_, pg) = (place(a, (first + i) % 4) for i, a in enumerate(base))
        out = [place(torch.zeros_like(t), (first + i) % 4) for i, t in enumerate((y, both) + grads)]
        ptr = [t.data_ptr() for _, t in out]
        ws, at, need = znn._take_workspace(px, max(znn.gated_workspace_bytes(f, fo, n, axis, p) for p in (0, 1)))
        assert L.znn_gated_fwd(3, f, fo, n, axis, px.data_ptr(), pw.data_ptr(), pb.data_ptr(), ptr[0], ptr[1], at, need, znn._stream_ptr()) == 0
        assert L.znn_gated_bwd(3, f, fo, n, axis, pg.data_ptr(), px.data_ptr(), pw.data_ptr(), ptr[1], ptr[2], ptr[3], ptr[4], at, need,
                               znn._stream_ptr()) == 0
        for i, ((held, t), want) in enumerate(zip(out, (y, both) + grads)):
            k = (first + i) % 4
            assert torch.equal(t, want), (first, i)
            assert bool((held[:k] == 7.5).all()) and bool((held[k + t.numel():] == 7.5).all()), (first, i)


@pytest.mark.parametrize("axis,shape,f,fo", [(0, (12, 12, 12), 40, 24), (1, (300,), 65, 40), (1, (1,), 200, 64), (1, (4, 5, 3), 64, 33)])
def test_calls_repeat_themselves_on_any_stream_and_in_a_graph(axis, shape, f, fo):
    n = int(np.prod(shape))
    x, w, b, gy = operands(f, fo, n, 23)
    view = lambda m, k: dev(lay(m, axis)).view(shape + (k,) if axis else (k,) + shape)  # noqa: E731
    x, gy, w, b = view(x, f), view(gy, fo), dev(w), dev(b)
    y, both = znn.gated_fwd(x, w, b, "gelu", axis)
    grads = znn.gated_bwd(gy, x, w, both, "gelu", axis)
    assert y.shape == gy.shape and grads[0].shape == x.shape and grads[1].shape == w.shape
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        a, k = znn.gated_fwd(x, w, b, "gelu", axis, stream=side)
        g = znn.gated_bwd(gy, x, w, k, "gelu", axis, stream=side)
        side.synchronize()
        assert torch.equal(a, y) and torch.equal(k, both) and all(torch.equal(p, q) for p, q in zip(g, grads))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, k = znn.gated_fwd(x, w, b, "gelu", axis)
        g = znn.gated_bwd(gy, x, w, k, "gelu", axis)
    for number in range(4):
        x.mul_(-1)
        gy.mul_(2)
        graph.replay()
        c, l = znn.gated_fwd(x, w, b, "gelu", axis)
        d = znn.gated_bwd(gy, x, w, l, "gelu", axis)
        torch.cuda.synchronize()
        assert torch.equal(a, c) and torch.equal(k, l) and all(torch.equal(p, q) for p, q in zip(g, d)), number


def test_what_nothing_reads_is_not_computed():
    x, w, b, gy = (dev(a) for a in operands(40, 24, 90, 29))
    y, both = znn.gated_fwd(x, w, b, "tanh")
    gx, gw, gb = znn.gated_bwd(gy, x, w, both, "tanh")
    none, gw2, gb2 = znn.gated_bwd(gy, x, w, both, "tanh", need_gx=False)
    assert none is None and torch.equal(gw, gw2) and torch.equal(gb, gb2)
    gx3, gw3, none = znn.gated_bwd(gy, x, w, both, "tanh", bias=False)
    assert none is None and torch.equal(gw, gw3) and torch.equal(gx, gx3)


def test_weights_of_a_convolution():
    """Weights as a layer with kernels of one voxel has them: the unit is that layer, its halves multiplied."""
    f, fo, n = 12, 10, (5, 6, 7)
    x, w, b, _ = operands(f, fo, int(np.prod(n)), 31)
    dx, dw, db = dev(x).view((f,) + n), dev(w).view(2 * fo, f, 1, 1, 1), dev(b)
    y, both = znn.gated_fwd(dx, dw, db, "logistic")
    plan = znn.Plan(f, 2 * fo, n, (1, 1, 1), "direct")
    layer = host(plan.fwd(dx, dw)) + b.astype(np.float64)[:, None, None, None]
    bound = 2 * gated.gated_fwd(x, w, b, "logistic")[3].reshape((2 * fo,) + n)
    assert np.all(np.abs(host(both) - layer) <= bound)
    assert znn.gated_bwd(dev(np.ones((fo,) + n)), dx, dw, both, "logistic")[1].shape == dw.shape


def test_gradients_against_differences():
    f, fo, n = 9, 7, 40
    x, w, b, gy = operands(f, fo, n, 37)
    r = np.random.default_rng(38)
    for fn in ("logistic", "tanh", "silu", "gelu"):
        _, both = znn.gated_fwd(dev(x), dev(w), dev(b), fn)
        grads = [host(g) for g in znn.gated_bwd(dev(gy), dev(x), dev(w), both, fn)]
        arrays = [t.astype(np.float64) for t in (x, w, b)]
        value = lambda x, w, b: (gated.gated_fwd(x, w, b, fn)[0] * gy).sum()  # noqa: E731
        for which in range(3):
            way = [np.zeros_like(t) for t in arrays]
            way[which] = r.normal(size=arrays[which].shape)
            e = 1e-5
            d = (value(*(t + e * v for t, v in zip(arrays, way))) - value(*(t - e * v for t, v in zip(arrays, way)))) / (2 * e)
            assert abs(d - (grads[which] * way[which]).sum()) <= 1e-5 * np.abs(grads[which] * way[which]).sum() + 1e-9
