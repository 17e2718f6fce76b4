"""Extents that take the kernels' remaining instances: features at and behind what every tile and every group of lanes holds, rows on
whole lines and not, with the parameters' gradients in the same launch and by shares.  Tolerances are those of test_gpu_norm.py."""
import numpy as np
import pytest
import torch

from oracle import net as onet
from oracle import norm
from paper_1510_06706_amd import binding as znn
from paper_1510_06706_amd import net as znet
from paper_1510_06706_amd import synth
from test_gpu_norm import EPS, SHARED, check_norm, get, put, test_layernorm as layernorm_case, test_residual_join as join_case

pytestmark = pytest.mark.gpu

ON_LINES = [(1, 64, 0), (3, 1024, 0), (16, 1024, 0), (17, 1024, 0), (24, 1024, 0), (32, 1024, 0), (33, 1024, 0), (64, 1024, 0), (65, 1024, 0),
            (120, 1024, 0), (128, 1024, 0), (129, 1024, 0), (200, 1024, 0), (256, 1024, 0), (300, 1024, 0), (512, 1024, 0), (16, 16384, 0),
            (24, 16384, 0), (32, 16384, 0), (48, 12320, 0), (120, 16384, 0), (200, 16384, 0), (300, 4096, 0)]
OFF_LINES = [(16, 1001, 0), (17, 1003, 0), (24, 1001, 0), (32, 1021, 0), (24, 16381, 0), (16, 13001, 0)]
# few rows by every number of lanes and quads, many by those of a workgroup
ROWS = [(64, 1024, 1), (512, 1025, 1), (64, 2049, 1), (64, 4100, 1), (64, 8195, 1), (64, 12289, 1), (64, 16000, 1), (1000, 12300, 1), (7, 16384, 1)]


@pytest.mark.parametrize("rows,cols,axis", ON_LINES + OFF_LINES + ROWS)
def test_norms(rows, cols, axis):
    layernorm_case(rows, cols, axis)


@pytest.mark.parametrize("p,use_gr", [(0.0, True), (0.3, False)])
@pytest.mark.parametrize("rows,cols,axis", ON_LINES + OFF_LINES + ROWS)
def test_joins(rows, cols, axis, p, use_gr):
    join_case(rows, cols, axis, p, use_gr)


@pytest.mark.parametrize("p,use_gr", [(0.0, True), (0.3, False), (0.0, False)])
@pytest.mark.parametrize("rows,cols,axis", SHARED)
def test_joins_that_leave_shares(rows, cols, axis, p, use_gr):
    join_case(rows, cols, axis, p, use_gr)


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("n", [130, 700, 17000])
def test_gradients_beside_a_mean_far_from_zero(axis, n):
    """The statistics hold the mean in 32 bits: (x - m) s is off by what was rounded of m, half an ulp of 4096, times s.  Gradients
    against statistics in 64 bits, with the tolerance that follows, beside the file's own."""
    rows, cols = (n, 67) if axis == 0 else (67, n)
    rs = np.random.RandomState(n)
    x = (rs.randn(rows, cols) + 4096).astype(np.float32)
    gy, w, b = rs.randn(rows, cols).astype(np.float32), (1 + 0.2 * rs.randn(n)).astype(np.float32), np.zeros(n, np.float32)
    tol = 64 * 2.0 ** -24
    y, stats = znn.layernorm_fwd(put(x), put(w), put(b), EPS, axis)
    check_norm(get(y), get(stats), x.astype(np.float64), w, b, axis)
    gx, gw, gb = (get(t) for t in znn.layernorm_bwd(put(gy), put(x), put(w), stats, axis))
    # positions along the second axis, in 64 bits
    turn = (lambda a: a) if axis == 1 else (lambda a: a.T)
    x, g, gx, w = turn(x.astype(np.float64)), turn(gy.astype(np.float64)), turn(gx), w.astype(np.float64)
    _, m, s = norm.layernorm_fwd(x, w, b, EPS, 1)
    m, s = m[:, None], s[:, None]
    h, a = (x - m) * s, g * w
    off = s * (np.spacing(np.float32(4096)) / 2 + tol * np.abs(x - m).mean(1, keepdims=True))
    want_gx, want_gw, want_gb = norm.layernorm_bwd(g, x, w, m[:, 0], s[:, 0], 1)
    mean_a, mean_ah = np.abs(a).mean(1, keepdims=True), np.abs(a * h).mean(1, keepdims=True)
    # the sums' roundings, and what s may be off by as a factor of the whole and twice in the last term
    rounding = 4 * tol * (np.abs(a) + mean_a + np.abs(h) * mean_ah)
    assert (np.abs(gx - want_gx) <= s * (rounding + off * mean_ah + (np.abs(h) + off) * off * mean_a)).all()
    assert (np.abs(gw - want_gw) <= 2 * tol * np.abs(g * h).sum(0) + (np.abs(g) * off).sum(0)).all()
    assert (np.abs(gb - want_gb) <= tol * np.abs(g).sum(0)).all()


@pytest.mark.parametrize("first", [("layernorm",), ("layernorm", 1e-2)])
def test_a_net_that_begins_with_a_norm(first):
    layers = [first, ("conv", 3, 4, (1, 3, 3)), ("transfer", "tanh"), ("layernorm",), ("conv", 4, 2, (1, 1, 1)), ("transfer", "logistic")]
    shape = (3, 2, 8, 9)
    params = synth.synthetic_params(layers, 6)
    x, target = synth.uniform_pm1(6, 0, shape), synth.uniform_01(6, 3, (2, 2, 6, 7))
    net = znet.Net(layers, shape, params, "direct")
    acts, _, _, grads = net.train_round(put(x), put(target), 0.0)
    p64 = [None if p is None else {k: v.astype(np.float64) for k, v in p.items()} for p in params]
    _, r_acts, _, r_grads, _ = onet.train_round(layers, p64, x, target, 0.0)
    for got, want in [(acts[-1], r_acts[-1])] + [(grads[l][k], g[k]) for l, g in enumerate(r_grads) for k in g or ()]:
        assert np.abs(get(got) - want).max() <= 1e-4 * np.abs(want).max()
    # prediction, and passes by hand
    assert torch.equal(net.forward(put(x))[0][-1], acts[-1])
    acts, aux = net.forward(put(x), train=True)
    by_hand = net.backward(acts, aux, znn.loss_grad(acts[-1], put(target)))
    for l, g in enumerate(r_grads):
        for k in g or ():
            assert np.abs(get(by_hand[l][k]) - g[k]).max() <= 1e-4 * np.abs(g[k]).max()
