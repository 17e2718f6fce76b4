"""Dropout, layer norm and the residual join on the GPU against the definitions in 64 bits.

Tolerances, in units of u = 2^-24 (half an ulp of 32 bits) and of the terms a result is the sum of: sums run in chains and
trees whose errors grow with the square root of their length, at most 64 of chained additions over the lengths here, each
further operation adds one u.  So 64 u times the sum of the magnitudes holds for sums, and for a result element 64 u times the
largest terms of its position.  What dropout gives is exact: one rounded product.
"""
import numpy as np
import pytest
import torch

from oracle import norm
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TOL = 64 * U
EPS = 1e-5
DEV = "cuda:0"

# (rows, cols, axis): positions and features of one, odd extents, rows that start at no round address, features just at and behind
# what a wave or a workgroup holds, few positions with many features and the other way round
SHAPES = [(1, 1, 0), (1, 1, 1), (1, 7, 0), (1, 7, 1), (6, 1, 0), (6, 1, 1), (3, 5, 0), (3, 5, 1),
          (40, 1728, 0), (37, 4099, 0), (120, 343, 0), (80, 61 * 17, 0), (257, 130, 0), (1030, 66, 0), (5, 20001, 0), (64, 64, 0), (16, 1, 0), (4200, 9, 0),
          (2, 70003, 0), (129, 3001, 0), (500, 1021, 0), (3, 262147, 0),
          (1, 1024, 1), (7, 63, 1), (64, 64, 1), (5, 255, 1), (5, 256, 1), (5, 257, 1), (33, 1001, 1), (16, 4096, 1), (3, 4097, 1), (9, 8200, 1),
          (2, 16385, 1), (2, 40003, 1), (1, 131075, 1), (2049, 24, 1), (70001, 3, 1), (5003, 130, 1), (1000, 513, 1), (300, 2047, 1)]
# what the shapes above leave out of the backward passes that add up shares: tiles of every height, on lines and not, rows by every number
# of lanes, and positions that no workgroup holds
SHARED = [(20, 12301, 0), (33, 16384, 0), (40, 12299, 0), (100, 13001, 0), (120, 12320, 0), (146, 12289, 0), (200, 12800, 0), (256, 12303, 0), (512, 1000, 0),
          # one to three columns in the last tile
          (30, 12419, 0), (40, 12354, 0), (100, 13057, 0), (300, 4099, 0), (2, 12545, 0),
          (600, 40, 1), (513, 100, 1), (700, 250, 1), (520, 500, 1), (700, 1500, 1), (1030, 3001, 1), (1025, 8000, 1), (1025, 9001, 1), (1025, 16383, 1),
          (513, 37, 0), (1024, 160, 0), (2047, 131, 0), (1100, 4097, 0), (3000, 4, 0), (5000, 3, 0), (700, 20001, 1)]


def arrays(rows, cols, axis, seed, *scales):
    rs = np.random.RandomState(seed)
    n = (rows, cols)[axis]
    out = [(rs.randn(rows, cols) * s).astype(np.float32) for s in scales]
    # features of their own offset; a position without a signal
    out[0] += (rs.randn(n) * 2).astype(np.float32).reshape((-1, 1) if axis == 0 else (1, -1))
    if axis == 0 and cols > 4:
        out[0][:, 3] = 0.25
    if axis == 1 and rows > 4:
        out[0][3] = 0.25
    w, b = (1 + 0.2 * rs.randn(n)).astype(np.float32), (0.2 * rs.randn(n)).astype(np.float32)
    return out, w, b


def put(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def get(t):
    return t.cpu().numpy().astype(np.float64)


def along(v, axis):
    return v[:, None] if axis == 0 else v[None, :]


def across(v, axis):
    return v[None, :] if axis == 0 else v[:, None]


def check_norm(y, stats, x, w, b, axis):
    """y and the statistics against those of x (what the call normalised, in 32 bits)."""
    want, m, s = norm.layernorm_fwd(x, w, b, EPS, axis)
    h = (x - across(m, axis)) * across(s, axis)
    w, b = w.astype(np.float64), b.astype(np.float64)
    top = np.abs(h).max(axis, keepdims=True)
    assert (np.abs(y - want) <= TOL * ((1 + top) * np.abs(along(w, axis)) + np.abs(along(b, axis)))).all()
    if stats is not None:
        assert (np.abs(stats[0] - m) <= TOL * np.abs(x).mean(axis)).all()
        assert (np.abs(stats[1] - s) <= TOL * s).all()


def check_gx(gx, gy, x, w, stats, axis, gr=None):
    """gx and, for the parameters, what they are the sums of."""
    want, ww, wb = norm.layernorm_bwd(gy, x, w, stats[0], stats[1], axis)
    m, s = across(stats[0], axis), across(stats[1], axis)
    h = (x - m) * s
    # (x - m) s is rounded by u of |h|, and what is rounded of m and s does not count: they are given
    a = np.abs(gy * along(w.astype(np.float64), axis))
    scale = np.abs(s) * (a + a.mean(axis, keepdims=True) + np.abs(h) * (a * np.abs(h)).mean(axis, keepdims=True))
    scale = np.broadcast_to(scale.max(axis, keepdims=True), x.shape)
    if gr is not None:
        want = want + gr
        scale = scale + np.abs(gr)
    assert (np.abs(gx - want) <= TOL * scale).all()
    return h, ww, wb


def check_grads(gx, gw, gb, gy, x, w, stats, axis, gr=None):
    h, ww, wb = check_gx(gx, gy, x, w, stats, axis, gr)
    other = 1 - axis
    assert (np.abs(gw - ww) <= TOL * np.abs(gy * h).sum(other)).all()
    assert (np.abs(gb - wb) <= TOL * np.abs(gy).sum(other)).all()


@pytest.mark.parametrize("rows,cols,axis", SHAPES + SHARED)
def test_layernorm(rows, cols, axis):
    (x, gy), w, b = arrays(rows, cols, axis, rows + cols, 1.0, 0.1)
    y, stats = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis)
    only, none = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis, stats=False)
    assert none is None and torch.equal(only, y)
    check_norm(get(y), get(stats), x.astype(np.float64), w, b, axis)
    got = znn.layernorm_bwd(put(gy), put(x), put(w), stats, axis)
    check_grads(*(get(t) for t in got), gy.astype(np.float64), x.astype(np.float64), w, get(stats), axis)
    again = znn.layernorm_bwd(put(gy), put(x), put(w), stats, axis)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("p,use_gr", [(0.0, True), (0.3, True), (0.3, False), (0.0, False)])
@pytest.mark.parametrize("rows,cols,axis", SHAPES)
def test_residual_join(rows, cols, axis, p, use_gr):
    (x, h, gy, gr), w, b = arrays(rows, cols, axis, 3 * rows + cols, 1.0, 0.5, 0.1, 0.1)
    state = znn.random_state(2 ** 63 + 12345)
    znn.random_advance(state)
    state = state if p else None
    r, y, stats = znn.residual_norm_fwd(put(h), put(x), put(w), put(b), p, state, 5, EPS, axis)
    f = norm.dropout_factor(rows, cols, p, 2 ** 63 + 12345, 1, 5).astype(np.float32)
    assert np.array_equal(r.cpu().numpy(), x + h * f)           # two roundings, as dropout and a node sum
    check_norm(get(y), get(stats), get(r), w, b, axis)
    r2, y2, none = znn.residual_norm_fwd(put(h), put(x), put(w), put(b), p, state, 5, EPS, axis, stats=False)
    assert none is None and torch.equal(r2, r) and torch.equal(y2, y)
    got = znn.residual_norm_bwd(put(gy), put(gr) if use_gr else None, r, put(w), stats, p, state, 5, axis)
    gx, gh, gw, gb = got
    check_grads(get(gx), get(gw), get(gb), gy.astype(np.float64), get(r), w, get(stats), axis, gr.astype(np.float64) if use_gr else None)
    assert np.array_equal(gh.cpu().numpy(), gx.cpu().numpy() * f)
    assert (gh is gx) == (p == 0)
    again = znn.residual_norm_bwd(put(gy), put(gr) if use_gr else None, r, put(w), stats, p, state, 5, axis)
    assert all(torch.equal(u, v) for u, v in zip(got, again))


@pytest.mark.parametrize("rows,cols,axis", SHARED)
def test_residual_join_with_shares(rows, cols, axis):
    test_residual_join(rows, cols, axis, 0.3, True)


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0, 1e-12])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (3, 1), (2, 5), (7, 64), (40, 1728), (36, 4987), (5, 1027), (4001, 2), (1, 70001)])
def test_dropout(rows, cols, p):
    x = np.random.RandomState(cols).randn(rows, cols).astype(np.float32)
    state = znn.random_state(987654321987654321)
    for number in range(2):
        y = znn.dropout(put(x), p, state, 7)
        f = norm.dropout_factor(rows, cols, p, 987654321987654321, number, 7).astype(np.float32)
        assert np.array_equal(y.cpu().numpy(), np.where(f > 0, x * f, np.float32(0)))
        znn.random_advance(state)
    assert state.cpu().tolist() == [987654321987654321, 2]
    if p == 0.0:
        assert torch.equal(znn.dropout(put(x), 0.0), put(x))


def test_what_a_dropped_element_holds_does_not_matter():
    f = norm.dropout_factor(4, 1001, 0.5, 9, 0, 0)
    x = np.where(f > 0, np.float32(1), np.float32("nan"))
    x[1] = np.where(f[1] > 0, 1, np.inf)
    x = x.astype(np.float32)
    state = znn.random_state(9)
    y = znn.dropout(put(x), 0.5, state).cpu().numpy()
    assert np.array_equal(y, f.astype(np.float32))
    for axis in (0, 1):
        n = x.shape[axis]
        one, zero = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
        r, out, _ = znn.residual_norm_fwd(put(x), put(np.ones_like(x)), one, zero, 0.5, state, axis=axis)
        assert np.array_equal(r.cpu().numpy(), 1 + f.astype(np.float32))
        assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("axis", [0, 1])
def test_positions_do_not_touch_each_other(axis):
    """NaN and infinity stay within their position, of which nothing is left that looks like a number."""
    (x, gy), w, b = arrays(96, 96, axis, 5, 1.0, 0.1)
    clean, stats = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis)
    gx0, _, _ = znn.layernorm_bwd(put(gy), put(x), put(w), stats, axis)
    bad = x.copy()
    spoil = bad if axis == 1 else bad.T
    spoil[10, 7], spoil[20, 50], spoil[30, 95] = np.nan, np.inf, -np.inf
    y, st = znn.layernorm_fwd(put(bad), put(w), put(b), EPS, axis)
    gx, _, _ = znn.layernorm_bwd(put(gy), put(bad), put(w), st, axis)
    hit = np.zeros(96, bool)
    hit[[10, 20, 30]] = True
    for got, want in ((y, clean), (gx, gx0)):
        got, want = (t.cpu().numpy() if axis == 1 else t.cpu().numpy().T for t in (got, want))
        assert np.isnan(got[hit]).all()
        assert np.array_equal(got[~hit], want[~hit])
    assert torch.isnan(st[:, put(hit)]).all()


@pytest.mark.parametrize("axis", [0, 1])
def test_means_far_from_zero(axis):
    """A deviation of 1 beside a mean of 4096 keeps the digits that the operand has."""
    (x,), w, b = arrays(130, 130, axis, 11, 1.0)
    x = (x + np.float32(4096)).astype(np.float32)
    y, stats = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis)
    check_norm(get(y), get(stats), x.astype(np.float64), w, b, axis)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("value", [0.0, 1.0, -3e30, 1e-30])
def test_constant_positions(axis, value):
    x = np.full((48, 48), value, np.float32)
    w, b = np.ones(48, np.float32), np.linspace(-1, 1, 48).astype(np.float32)
    y, stats = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis)
    # powers of two times a sum of 48 equal values are exact up to three bits: the mean is the value but for its last ones
    assert bool(torch.isfinite(y).all()) and bool(torch.isfinite(stats).all())
    if abs(value) <= 1:
        assert (np.abs(get(y) - along(b.astype(np.float64), axis)) <= TOL * (1 + abs(value) * EPS ** -0.5)).all()


@pytest.mark.parametrize("axis", [0, 1])
def test_gradients_against_differences(axis):
    """Along one direction, from what the forward call itself gives: steps of e and 2 e leave an error of e^4."""
    rows, cols = 37, 53
    (x, h, gy, gr, v), w, b = arrays(rows, cols, axis, 21, 1.0, 1.0, 1.0, 1.0, 1.0)
    v -= along(v.mean(1 - axis), axis)
    state, p = znn.random_state(4), 0.4
    dw, db = np.random.RandomState(3).randn(2, w.size).astype(np.float32)

    def value(e, which):
        m = lambda a, d, name: put((a + np.float32(e) * d).astype(np.float32) if which == name else a)  # noqa: E731
        r, y, _ = znn.residual_norm_fwd(m(h, v, "h"), m(x, v, "x"), m(w, dw, "w"), m(b, db, "b"), p, state, 1, EPS, axis)
        return float((get(y) * gy + get(r) * gr).sum())

    r, _, stats = znn.residual_norm_fwd(put(h), put(x), put(w), put(b), p, state, 1, EPS, axis)
    gx, gh, gw, gb = znn.residual_norm_bwd(put(gy), put(gr), r, put(w), stats, p, state, 1, axis)
    e = 2.0 ** -6
    for which, got, d in (("x", gx, v), ("h", gh, v), ("w", gw, dw), ("b", gb, db)):
        slope = (8 * (value(e, which) - value(-e, which)) - (value(2 * e, which) - value(-2 * e, which))) / (12 * e)
        terms = np.abs(get(got) * d).sum()
        # rounding: about 2000 values of 2 u each at random signs over e, i.e. 45 * 4 u / e; the fourth order: deviations here are above 0.7
        # but for the position without a signal of its own, which x + dropout(h) gives one
        assert abs(slope - float((get(got) * d).sum())) <= 2e-3 * terms, which


def test_a_stream_of_the_caller():
    (x, h, gy, gr), w, b = arrays(64, 3001, 0, 2, 1.0, 1.0, 1.0, 1.0)
    state = znn.random_state(1)
    t = [put(a) for a in (x, h, gy, gr, w, b)]
    tx, th, tgy, tgr, tw, tb = t

    def all_of(stream):
        d = znn.dropout(tx, 0.2, state, 0, stream=stream)
        y, st = znn.layernorm_fwd(tx, tw, tb, EPS, 0, stream=stream)
        back = znn.layernorm_bwd(tgy, tx, tw, st, 0, stream=stream)
        r, y2, st2 = znn.residual_norm_fwd(th, tx, tw, tb, 0.2, state, 0, EPS, 0, stream=stream)
        return [d, y, st, *back, r, y2, st2, *znn.residual_norm_bwd(tgy, tgr, r, tw, st2, 0.2, state, 0, 0, stream=stream)]

    want = all_of(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = all_of(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_recorded_calls_draw_new_masks_at_every_replay():
    (x, h, gy, gr), w, b = arrays(40, 1000, 0, 8, 1.0, 1.0, 1.0, 1.0)
    tx, th, tgy, tgr, tw, tb = (put(a) for a in (x, h, gy, gr, w, b))
    state, eager = znn.random_state(6), znn.random_state(6)

    def round_of(state):
        r, y, st = znn.residual_norm_fwd(th, tx, tw, tb, 0.3, state, 2, EPS, 0)
        out = [r, y, st, *znn.residual_norm_bwd(tgy, tgr, r, tw, st, 0.3, state, 2, 0), znn.dropout(tx, 0.3, state, 3)]
        znn.random_advance(state)
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        round_of(znn.random_state(0))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = round_of(state)
    seen = []
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = round_of(eager)
        assert all(torch.equal(a, b) for a, b in zip(recorded, want))
        seen.append(recorded[0].clone())
        torch.cuda.synchronize()
    assert all(not torch.equal(seen[0], s) for s in seen[1:])
    assert state.cpu().tolist() == [6, 4]


def test_unaligned_operands():
    """Operands that start at any element, and rows of no round length behind them."""
    for rows, cols, axis in ((5, 66, 1), (20, 1001, 0)):
        n = (rows, cols)[axis]
        make = lambda c, k: torch.randn(c + k, generator=torch.Generator().manual_seed(c + k)).to(DEV)[k:]  # noqa: E731
        x, h, gy = (make(rows * cols, k).view(rows, cols) for k in (1, 2, 3))
        w, b = make(n, 1), make(n, 3)
        assert x.data_ptr() % 16 == 4
        state = znn.random_state(3)
        same = [t.clone() for t in (h, x, w, b, gy)]
        r, y, st = znn.residual_norm_fwd(h, x, w, b, 0.2, state, 0, EPS, axis)
        r2, y2, st2 = znn.residual_norm_fwd(*same[:4], 0.2, state, 0, EPS, axis)
        assert torch.equal(r, r2) and torch.equal(y, y2) and torch.equal(st, st2)
        a, c = znn.residual_norm_bwd(gy, None, r, w, st, 0.2, state, 0, axis), znn.residual_norm_bwd(same[4], None, r, same[2], st, 0.2, state, 0, axis)
        assert all(torch.equal(u, v) for u, v in zip(a, c))


def test_offsets_behind_32_bits():
    """2^31 elements and more: the last rows and columns of a large array."""
    rows, cols = 3, (1 << 30) + 6
    x = torch.ones(rows * cols, device=DEV).view(rows, cols)
    state = znn.random_state(5)
    y = znn.dropout(x, 0.5, state, 1)
    first = (1 << 30) - 2000
    want = norm.dropout_factor(1, cols - first, 0.5, 5, 0, 1, first_row=2, first_col=first)
    assert np.array_equal(get(y[2:, first:]), want)
    del y
    for axis, shape in ((0, (129, 16700001)), (1, (16700001, 129))):
        a = x.view(-1)[:shape[0] * shape[1]].view(shape)
        tail = (slice(None), slice(-70, None)) if axis == 0 else (slice(-70, None), slice(None))
        part = np.random.RandomState(1).randn(*a[tail].shape).astype(np.float32)
        a[tail] = put(part)
        w, b = torch.full((129,), 2.0, device=DEV), torch.full((129,), 0.5, device=DEV)
        yy, st = znn.layernorm_fwd(a, w, b, EPS, axis)
        check_norm(get(yy[tail]), get(st[:, -70:]), part.astype(np.float64), get(w).astype(np.float32), get(b).astype(np.float32), axis)
        assert bool((yy[:, 0] == 0.5).all() if axis == 0 else (yy[0] == 0.5).all())
        gx, gw, gb = znn.layernorm_bwd(yy, a, w, st, axis)
        # a position's gradient along its own result is the small difference of large terms: held to those, as everywhere
        check_gx(get(gx[tail]), get(yy[tail]), part.astype(np.float64), get(w), get(st[:, -70:]), axis)
        del yy, gx


@pytest.mark.parametrize("change,error", [
    (dict(x=lambda t: t.t()), ValueError), (dict(x=lambda t: t.double()), ValueError), (dict(x=lambda t: t.cpu()), ValueError),
    (dict(h=lambda t: t[:, :-1].contiguous()), ValueError), (dict(w=lambda t: t[:-1]), ValueError), (dict(b=lambda t: t.half()), ValueError),
    (dict(axis=2), ValueError), (dict(p=1.5, ), znn.ZnnError), (dict(p=0.5, state=None), znn.ZnnError), (dict(eps=0.0), znn.ZnnError),
    (dict(state=lambda t: t[:1]), ValueError), (dict(state=lambda t: t.int()), ValueError)])
def test_what_the_calls_refuse(change, error):
    args = dict(h=torch.zeros(6, 8, device=DEV), x=torch.zeros(6, 8, device=DEV), w=torch.zeros(6, device=DEV), b=torch.zeros(6, device=DEV),
                p=0.5, state=znn.random_state(0), eps=1e-5, axis=0)
    args.update({k: v(args[k]) if callable(v) else v for k, v in change.items()})
    with pytest.raises(error):
        znn.residual_norm_fwd(**args)
