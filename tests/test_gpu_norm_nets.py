"""Layer norm and dropout as layers of nets and edges of graphs: rounds against the reference in 64 bits, recorded rounds,
passes by hand, and rounds on several streams."""
import numpy as np
import pytest
import torch

from oracle import graph as ograph
from oracle import net as onet
from oracle import norm
from paper_1510_06706_amd import binding as znn
from paper_1510_06706_amd import graph as zgraph
from paper_1510_06706_amd import net as znet
from paper_1510_06706_amd import synth

pytestmark = pytest.mark.gpu

SEED = 91
# smooth transfer functions: no rectifier that rounding may open or close
LAYERS = [("conv", 1, 12, (3, 3, 3)), ("layernorm",), ("transfer", "tanh"), ("dropout", 0.3),
          ("conv", 12, 10, (3, 3, 3)), ("transfer", "tanh"), ("dropout", 0.0), ("layernorm", 1e-3), ("maxfilter", (2, 2, 2)), ("dropout", 0.1),
          ("conv", 10, 2, (2, 2, 2)), ("transfer", "logistic")]
IN_SHAPE = (1, 13, 14, 12)
# direct and FFT method, as for whole nets elsewhere; the norms' own errors are a thousand times smaller
TOLERANCE = {"direct": 1e-4, "fft": 1e-3}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")


def host(t):
    return t.cpu().numpy().astype(np.float64)


def rel_err(a, r):
    return float(np.max(np.abs(a - r)) / np.max(np.abs(r)))


def net_factors(layers, shapes, number):
    return {l: norm.dropout_factor(shapes[l][0], int(np.prod(shapes[l][1:])), s[1], SEED, number, l).reshape(shapes[l])
            for l, s in enumerate(layers) if s[0] == "dropout"}


def wide(params):
    return [None if p is None else {k: v.astype(np.float64) for k, v in p.items()} for p in params]


@pytest.mark.parametrize("mode", ["direct", "fft"])
def test_rounds_of_a_net(mode):
    x, target, params = synth.net_tensors(LAYERS, IN_SHAPE, 17)
    shapes = synth.shapes(LAYERS, IN_SHAPE)
    net = znet.Net(LAYERS, IN_SHAPE, params, mode, seed=SEED)
    by_layer = znet.Net(LAYERS, IN_SHAPE, params, mode, seed=SEED)
    p64 = wide(params)
    for number in range(3):
        acts, aux, gout, grads = net.train_round(dev(x), dev(target), 0.05)
        factors = net_factors(LAYERS, shapes, number)
        _, r_acts, r_aux, r_grads, p64 = onet.train_round(LAYERS, p64, x, target, 0.05, factors=factors)
        for l, spec in enumerate(LAYERS):
            assert rel_err(host(acts[l + 1]), r_acts[l + 1]) <= TOLERANCE[mode], (number, l)
            if spec[0] == "dropout" and spec[1] > 0:
                assert np.array_equal(host(acts[l + 1]) == 0, (factors[l] == 0) | (host(acts[l]) == 0))
        # the same voxels chosen by the max-filter, or gradients differ by whole terms
        assert np.array_equal(host(aux[8]), r_aux[8])
        for l, g in enumerate(r_grads):
            for k in g or ():
                assert rel_err(host(grads[l][k]), g[k]) <= TOLERANCE[mode], (number, l, k)
                assert rel_err(host(net.params[l][k]), p64[l][k]) <= TOLERANCE[mode], (number, l, k)
        # one library call per layer: the same operations, sums in another order here and there
        acts1, _, _, grads1 = by_layer.train_round(dev(x), dev(target), 0.05, record=[])
        assert rel_err(host(acts1[-1]), host(acts[-1])) <= 1e-5
        for l, g in enumerate(grads1):
            for k in g or ():
                assert rel_err(host(g[k]), host(grads[l][k])) <= 1e-4, (l, k)
    assert net.random.cpu().tolist() == by_layer.random.cpu().tolist() == [SEED, 3]


def test_predictions_drop_nothing():
    x, _, params = synth.net_tensors(LAYERS, IN_SHAPE, 18)
    net = znet.Net(LAYERS, IN_SHAPE, params, "direct", seed=SEED)
    acts, _ = net.forward(dev(x))
    want, _ = onet.forward(LAYERS, wide(params), x)
    for a, w in zip(acts, want):
        assert rel_err(host(a), w) <= TOLERANCE["direct"]
    assert acts[4] is acts[3] and net.random.cpu().tolist() == [SEED, 0]


def test_a_net_that_begins_with_dropout():
    layers = [("dropout", 0.5), ("conv", 2, 3, (1, 3, 3)), ("layernorm",), ("transfer", "tanh")]
    shape = (2, 1, 9, 11)
    params = synth.synthetic_params(layers, 4)
    x, target = synth.uniform_pm1(4, 0, shape), synth.uniform_01(4, 3, (3, 1, 7, 9))
    net = znet.Net(layers, shape, params, "direct", seed=SEED)
    acts, _ = net.forward(dev(x))
    assert rel_err(host(acts[-1]), onet.forward(layers, wide(params), x)[0][-1]) <= 1e-4
    _, _, _, grads = net.train_round(dev(x), dev(target), 0.0)
    want = onet.train_round(layers, wide(params), x, target, 0.0, factors=net_factors(layers, synth.shapes(layers, shape), 0))[3]
    for l, g in enumerate(want):
        for k in g or ():
            assert rel_err(host(grads[l][k]), g[k]) <= 1e-4, (l, k)


def test_passes_by_hand_give_a_rounds_gradients():
    x, target, params = synth.net_tensors(LAYERS, IN_SHAPE, 19)
    net = znet.Net(LAYERS, IN_SHAPE, params, "direct", seed=SEED)
    acts, aux = net.forward(dev(x), train=True)
    grads = net.backward(acts, aux, znn.loss_grad(acts[-1], dev(target)))
    again = znet.Net(LAYERS, IN_SHAPE, params, "direct", seed=SEED).train_round(dev(x), dev(target), 0.0)[3]
    for l, g in enumerate(grads):
        for k in g or ():
            assert rel_err(host(g[k]), host(again[l][k])) <= 1e-4, (l, k)


def test_recorded_rounds_are_eager_ones():
    x, target, params = synth.net_tensors(LAYERS, IN_SHAPE, 20)
    net, eager = (znet.Net(LAYERS, IN_SHAPE, params, "direct", seed=SEED) for _ in range(2))
    dx, dt = dev(x), dev(target)
    replay, (acts, _, _, grads) = net.capture_round(dx, dt, 0.02)
    assert net.random.cpu().tolist() == [SEED, 0]
    dropped = []
    for number in range(4):
        replay()
        torch.cuda.synchronize()
        want = eager.train_round(dx, dt, 0.02)
        assert all(torch.equal(a, b) for a, b in zip(acts[1:], want[0][1:]))
        for l, p in enumerate(net.params):
            for k in p or ():
                assert torch.equal(p[k], eager.params[l][k]) and torch.equal(grads[l][k], want[3][l][k]), (number, l, k)
        dropped.append(acts[4] == 0)
        dropped[-1] = dropped[-1].clone()
    assert all(not torch.equal(dropped[0], d) for d in dropped[1:])


def residual_graph(width=8, n=12):
    """A first layer, then two residual branches of 1 x 1 x 1 kernels that dropout ends; every sum is normalised."""
    k1, k3 = (1, 1, 1), (3, 3, 3)
    edges = [("conv", "c0", "x", "a", width, k3)]
    at = "a"
    for i in range(2):
        b = str(i)
        edges += [("layernorm", "n" + b, at, "h" + b), ("conv", "u" + b, "h" + b, "p" + b, 2 * width, k1), ("transfer", "t" + b, "p" + b, "q" + b, "tanh"),
                  ("conv", "d" + b, "q" + b, "r" + b, width, k1), ("dropout", "o" + b, "r" + b, "s" + b, 0.25), ("dropout", "i" + b, at, "s" + b, 0.0)]
        at = "s" + b
    edges += [("layernorm", "n", at, "f", 1e-4), ("conv", "c1", "f", "o", 2, k3), ("transfer", "t", "o", "y", "logistic")]
    return {"inputs": {"x": (1, n, n, n)}, "edges": edges, "outputs": ["y"]}


def test_rounds_of_a_graph_with_residual_branches():
    g = residual_graph()
    inputs, targets, params = synth.graph_tensors(g, 31)
    shapes = synth.graph_shapes(g)
    di, dt = {n: dev(v) for n, v in inputs.items()}, {n: dev(v) for n, v in targets.items()}
    nets = [zgraph.GraphNet(g, params, "direct", streams=s, seed=SEED) for s in (None, 1, 4)]
    p64 = {n: {k: v.astype(np.float64) for k, v in p.items()} for n, p in params.items()}
    order = [e[1] for e in zgraph.edge_order(g)]
    for number in range(2):
        factors = {}
        for e in g["edges"]:
            if e[0] == "dropout" and e[4] > 0:
                s = shapes[e[2]]
                factors[e[1]] = norm.dropout_factor(s[0], int(np.prod(s[1:])), e[4], SEED, number, order.index(e[1])).reshape(s)
        # passes by hand first: they leave the state as it is
        img1, aux1, _ = nets[0].forward(di, train=True)
        grads1, _ = nets[0].backward(img1, aux1, {"y": znn.loss_grad(img1["y"], dt["y"], "cross_entropy")})
        results = [net.train_round(di, dt, 1e-3, "cross_entropy") for net in nets]
        _, r_img, _, r_grads, p64 = ograph.train_round(g, p64, inputs, targets, 1e-3, "cross_entropy", factors)
        img, _, _, grads = results[0]
        for n in r_img:
            assert rel_err(host(img[n]), r_img[n]) <= 1e-4, (number, n)
        for n, d in r_grads.items():
            for k in d:
                assert rel_err(host(grads[n][k]), d[k]) <= 1e-4, (number, n, k)
                assert rel_err(host(grads1[n][k]), d[k]) <= 1e-4, (number, n, k)
                assert all(torch.equal(grads[n][k], r[3][n][k]) for r in results[1:]), (number, n, k)
    assert all(net.random.cpu().tolist() == [SEED, 2] for net in nets)
    plain = nets[0].forward(di)[0]
    want = ograph.forward(g, {n: {k: host(v) for k, v in p.items()} for n, p in nets[0].params.items()}, inputs)[0]
    torch.cuda.synchronize()
    assert rel_err(host(plain["y"]), want["y"]) <= 1e-4


def test_the_end_of_a_branch_is_one_operation():
    """Dropout, the sum with what passes the branch by, and the norm behind it; backward, the norm adds the other gradient."""
    from paper_1510_06706_amd import program as zp
    g = residual_graph()
    inputs, targets, params = synth.graph_tensors(g, 32)
    net = zgraph.GraphNet(g, params, "direct", seed=SEED)
    net.train_round({n: dev(v) for n, v in inputs.items()}, {n: dev(v) for n, v in targets.items()}, 0.0)
    kinds = [op["kind"] for op in net._programs["square"][0].ops]
    assert kinds.count(zp.JOIN_FWD) == 2 and kinds.count(zp.NODE_SUM) == 0
    assert kinds.count(zp.NORM_FWD) == 1 and kinds.count(zp.NORM_BWD) == 3
    assert kinds.count(zp.DROPOUT) == 2                 # backward
    assert sum(op["kind"] == zp.NORM_BWD and op["buf"][7] >= 0 for op in net._programs["square"][0].ops) == 2


def test_joins_that_lead_to_a_sum_and_to_two_norms():
    """A join whose norm ends in a node with another edge, beside a second norm of the same node, which is an output too."""
    k1 = (1, 1, 1)
    g = {"inputs": {"x": (3, 2, 5, 6)},
         "edges": [("conv", "c", "x", "h", 4, k1), ("conv", "c2", "x", "a", 4, k1), ("dropout", "d", "h", "s", 0.4), ("dropout", "i", "a", "s", 0.0),
                   ("layernorm", "n", "s", "u"), ("layernorm", "m", "s", "v", 1e-2), ("conv", "e", "a", "u", 4, k1), ("conv", "f", "v", "u", 4, k1),
                   ("transfer", "t", "u", "y", "tanh")],
         "outputs": ["y", "s"]}
    inputs, targets, params = synth.graph_tensors(g, 33)
    p64 = {n: {k: v.astype(np.float64) for k, v in p.items()} for n, p in params.items()}
    nets = [zgraph.GraphNet(g, params, "direct", streams=s, seed=SEED) for s in (None, 3)]
    site = [e[1] for e in zgraph.edge_order(g)].index("d")
    factors = {"d": norm.dropout_factor(4, 60, 0.4, SEED, 0, site).reshape(4, 2, 5, 6)}
    _, r_img, _, r_grads, _ = ograph.train_round(g, p64, inputs, targets, 0.0, "square", factors)
    results = [net.train_round({n: dev(v) for n, v in inputs.items()}, {n: dev(v) for n, v in targets.items()}, 0.0) for net in nets]
    for img, _, _, grads in results:
        for n in r_img:
            assert rel_err(host(img[n]), r_img[n]) <= 1e-4, n
        for n, d in r_grads.items():
            for k in d:
                assert rel_err(host(grads[n][k]), d[k]) <= 1e-4, (n, k)


@pytest.mark.parametrize("p", [-0.1, 1.0, 1.5, float("nan")])
def test_probabilities_that_nets_refuse(p):
    layers = [("conv", 1, 2, (1, 1, 1)), ("dropout", p), ("transfer",)]
    with pytest.raises(ValueError):
        znet.Net(layers, (1, 2, 2, 2), synth.synthetic_params(layers, 1), "direct")
    g = {"inputs": {"x": (1, 2, 2, 2)}, "edges": [("dropout", "d", "x", "y", p)], "outputs": ["y"]}
    with pytest.raises(ValueError):
        zgraph.GraphNet(g, {}, "direct")
