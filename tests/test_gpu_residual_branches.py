"""Residual nets with gated branches and with recurrences along the lines of the volume: rounds against the definitions in 64 bits,
predictions, recorded rounds, gradients."""
import numpy as np
import pytest
import torch

from oracle import gated, norm
from paper_1510_06706_amd import residual, synth

pytestmark = pytest.mark.gpu

SEED = 404


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")


def host(t):
    return t.cpu().numpy().astype(np.float64)


def rel_err(a, r):
    return float(np.max(np.abs(a - r)) / np.max(np.abs(r)))


def as_lines(t, extents, kind):
    """[maps][voxels] -> [outer][length][inner] along the branch's axis"""
    d = residual.LINES[kind]
    t = t.reshape((t.shape[0],) + extents)
    return t.reshape(int(np.prod(t.shape[:d])), t.shape[d], -1)


class Plain:
    """One round of the net on matrices [maps][voxels] in 64 bits."""

    def __init__(self, kinds, gate, extents, params, p, fn):
        self.kinds, self.gate, self.extents, self.p, self.fn = kinds, gate, extents, p, fn
        self.params = {k: (v.reshape(v.shape[0], -1) if v.ndim == 5 else v).astype(np.float64) for k, v in params.items()}

    def factor(self, maps, number, site):
        return norm.dropout_factor(maps, int(np.prod(self.extents)), self.p, SEED, number, site)

    def branch(self, i, y):
        q, kind = self.params, self.kinds[i - 1]
        a = q["w1_%d" % i] @ y
        if kind in residual.LINES:
            z0, x0, z1, x1 = (as_lines(t, self.extents, kind) for t in np.split(a, 4))
            h = [gated.recurrence_fwd(z0, x0, None, False)[0], gated.recurrence_fwd(z1, x1, None, True)[0]]
            return np.concatenate([t.reshape(a.shape[0] // 4, -1) for t in h]), a
        a = a + q["b1_%d" % i][:, None]
        if kind == "gated":
            u, v = np.split(a, 2)
            return gated.gate_fn(u, self.gate)[0] * v, a
        return gated.gate_fn(a, self.fn)[0], a

    def round(self, x, target, number, drops=True):
        q, n = self.params, len(self.kinds)
        keep = [self.factor(x.shape[0], number, i) if drops else 1.0 for i in range(n + 1)]
        r = x * keep[0]
        held = []
        for i in range(n + 1):
            if i:
                res, a = self.branch(i, y)
                h = q["w2_%d" % i] @ res
                r = r + h * keep[i]
                held[-1] += (res, a)
            y, m, s = norm.layernorm_fwd(r, q["norm_w_%d" % i], q["norm_b_%d" % i], 1e-5, 0)
            held.append((r, y, m, s))
        out = gated.sigmoid(q["w"] @ y + q["b"][:, None])
        g = out - target            # cross-entropy and logistic together
        grads = {"w": g @ y.T, "b": g.sum(1)}
        gy, gr = q["w"].T @ g, 0.0
        for i in range(n, -1, -1):
            r, y, m, s = held[i][:4]
            gx, grads["norm_w_%d" % i], grads["norm_b_%d" % i] = norm.layernorm_bwd(gy, r, q["norm_w_%d" % i], m, s, 0)
            gr = gx + gr
            if i == 0:
                break
            below, (res, a), kind = held[i - 1][1], held[i - 1][4:], self.kinds[i - 1]
            gh = gr * keep[i]
            grads["w2_%d" % i] = gh @ res.T
            gres = q["w2_%d" % i].T @ gh
            if kind == "gated":
                u, v = np.split(a, 2)
                f, d = gated.gate_fn(u, self.gate)
                ga = np.concatenate([gres * v * d, gres * f])
            elif kind == "plain":
                ga = gres * gated.gate_fn(a, self.fn)[1]
            else:
                z0, x0, z1, x1 = (as_lines(t, self.extents, kind) for t in np.split(a, 4))
                (g0, g1), (h0, h1) = ([as_lines(t, self.extents, kind) for t in np.split(b, 2)] for b in (gres, res))
                parts = gated.recurrence_bwd(g0, z0, x0, h0, None, False)[0][:2] + gated.recurrence_bwd(g1, z1, x1, h1, None, True)[0][:2]
                ga = np.concatenate([t.reshape(a.shape[0] // 4, -1) for t in parts])
            if kind not in residual.LINES:
                grads["b1_%d" % i] = ga.sum(1)
            grads["w1_%d" % i] = ga @ below.T
            gy = q["w1_%d" % i].T @ ga
        return out, grads


NETS = [(6, 10, ("gated",), 2, (3, 7, 9)), (5, 4, ("lines_x", "gated"), 1, (4, 6, 33)), (7, 6, ("lines_z", "lines_y", "lines_x"), 2, (12, 9, 10)),
        (33, 20, ("plain", "lines_y", "gated", "plain"), 3, (1, 30, 11))]


@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("maps,hidden,kinds,out_maps,extents", NETS)
def test_rounds(maps, hidden, kinds, out_maps, extents, p):
    gate = ["silu", "gelu", "logistic", "tanh"][maps % 4]
    params = residual.residual_params(maps, hidden, len(kinds), out_maps, 7, kinds)
    x = synth.uniform_pm1(3, 0, (maps,) + extents)
    target = synth.uniform_01(3, 3, (out_maps,) + extents)
    net = residual.ResidualNet(maps, hidden, len(kinds), out_maps, extents, params, p, "tanh", "direct", seed=SEED, branches=kinds, gate=gate)
    ref = Plain(kinds, gate, extents, params, p, "tanh")
    mx, mt = x.reshape(maps, -1).astype(np.float64), target.reshape(out_maps, -1).astype(np.float64)
    assert rel_err(host(net.forward(dev(x))).reshape(out_maps, -1), ref.round(mx, mt, 0, False)[0]) <= 1e-4
    for number in range(2):
        want, grads = ref.round(mx, mt, number)
        out, got = net.train_round(dev(x), dev(target), 1e-3)
        assert rel_err(host(out).reshape(out_maps, -1), want) <= 1e-4
        assert set(got) == set(grads)
        for k, g in grads.items():
            assert rel_err(host(got[k]).reshape(g.shape), g) <= 1e-4, (number, k)
            ref.params[k] = ref.params[k] - 1e-3 * g
            assert rel_err(host(net.params[k]).reshape(g.shape), ref.params[k]) <= 1e-4, (number, k)
    assert net.random.cpu().tolist() == [SEED, 2]


def test_recorded_rounds():
    maps, extents, kinds = 16, (6, 16, 18), ("lines_x", "gated", "lines_z")
    params = residual.residual_params(maps, 24, 3, 1, 9, kinds)
    x, target = synth.uniform_pm1(5, 0, (maps,) + extents), synth.uniform_01(5, 3, (1,) + extents)
    net, eager = (residual.ResidualNet(maps, 24, 3, 1, extents, params, 0.1, seed=SEED, branches=kinds) for _ in range(2))
    dx, dt = dev(x), dev(target)
    replay, (out, grads) = net.capture_round(dx, dt, 1e-4)
    for number in range(4):
        replay()
        torch.cuda.synchronize()
        want, wgrads = eager.train_round(dx, dt, 1e-4)
        assert torch.equal(out, want) and all(torch.equal(grads[k], wgrads[k]) for k in wgrads), number
        assert all(torch.equal(net.params[k], eager.params[k]) for k in params), number


def test_what_lines_bring_to_a_voxel():
    """A change at one voxel reaches the whole of its lines, and nothing else, in a net with one branch along them."""
    maps, extents = 6, (5, 6, 7)
    x = synth.uniform_pm1(5, 0, (maps,) + extents)
    for kind, d in residual.LINES.items():
        net = residual.ResidualNet(maps, 8, 1, 1, extents, residual.residual_params(maps, 8, 1, 1, 9, (kind,)), 0.0, branches=(kind,))
        a = net.forward(dev(x))
        x2 = x.copy()
        x2[0, 2, 3, 4] += 1         # of one map: what all have in common the norm takes away
        changed = (net.forward(dev(x2)) != a)[0].cpu().numpy()
        line = [2, 3, 4]
        line[d - 1] = slice(None)
        assert changed[tuple(line)].all()
        changed[tuple(line)] = False
        assert not changed.any()
