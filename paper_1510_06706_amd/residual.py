"""A residual net over the maps of every voxel, trained through the C ABI: what is put on the features of a
convolutional net to predict labels per voxel.

    r_0 = dropout(x),  y_0 = norm_0(r_0)
    r_i = r_(i-1) + dropout(W2_i branch_i(y_(i-1))),  y_i = norm_i(r_i)          i = 1 .. blocks
    out = logistic(W y_blocks + b)

A branch is one of
    "plain"       f(W1 y + b)
    "gated"       fn(U y + b) (V y + c), the two halves of W1 with 2 hidden rows: the gated unit
    "lines_z", "lines_y", "lines_x"   what a voxel sees along its line of the volume: W1 with 4 hidden rows makes gates and operands of two
                  gated recurrences along that axis, one from either end, whose states are the 2 hidden maps of the branch
so that a net without the last kind labels every voxel by itself, and one with them by all the voxels that its lines reach.

The products are convolutions with 1 x 1 x 1 kernels; the gated unit is one library call in each direction, a recurrence is one, and so is the end of every
branch - dropout, node sum and the norm that the next block begins with.  Images keep their extents, so the net fits any volume.
This module only sequences library calls; every arithmetic step runs in libznn's kernels.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as znn
from .synth import ONES, STREAM_BIAS, STREAM_KERNEL, uniform_pm1


LINES = {"lines_z": 1, "lines_y": 2, "lines_x": 3}      # the dimension of an image that a branch's lines run along


def _kinds(blocks, branches):
    kinds = ("plain",) * blocks if branches is None else tuple(branches)
    if len(kinds) != blocks:
        raise ValueError("expected %d branches, got %r" % (blocks, branches))
    for kind in kinds:
        if kind not in ("plain", "gated") and kind not in LINES:
            raise ValueError("a branch is plain, gated, %s, got %r" % (", ".join(LINES), kind))
    return kinds


def residual_params(maps, hidden, blocks, out_maps, seed, branches=None):
    """Seeded fp32 parameters by name, in the distributions of ``synth.synthetic_params``; ``branches``: the kind of every block's."""
    p = {}
    kinds = _kinds(blocks, branches)

    def kernels(name, f, fo):
        p[name] = uniform_pm1(seed + 17 * len(p), STREAM_KERNEL, (fo, f) + ONES, float(np.sqrt(6.0 / f)))

    def small(name, n, around=0.0):
        p[name] = np.float32(around) + uniform_pm1(seed + 17 * len(p), STREAM_BIAS, (n,), 0.1)

    for i in range(blocks + 1):
        if i > 0:
            kind = kinds[i - 1]
            kernels("w1_%d" % i, maps, 4 * hidden if kind in LINES else 2 * hidden if kind == "gated" else hidden)
            if kind not in LINES:       # the norm's own bias is one for gates and operands
                small("b1_%d" % i, 2 * hidden if kind == "gated" else hidden)
            kernels("w2_%d" % i, 2 * hidden if kind in LINES else hidden, maps)
        small("norm_w_%d" % i, maps, 1.0)
        small("norm_b_%d" % i, maps)
    kernels("w", maps, out_maps)
    small("b", out_maps)
    return p


class ResidualNet:
    """``params`` as ``residual_params`` names them.  ``p`` is the probability to drop in training rounds; what is dropped
    follows from ``random``, the device's {seed, round}, which a round moves on by one.  ``branches`` says what kind every block's is
    (None: all plain), ``gate`` which function gates the gated ones."""

    def __init__(self, maps, hidden, blocks, out_maps, extents, params, p=0.1, fn="rectify", mode="auto", eps=znn.NORM_EPS, seed=0,
                 device="cuda:0", branches=None, gate="silu"):
        self.maps, self.blocks, self.p, self.fn, self.eps = maps, blocks, float(p), fn, eps
        self.kinds, self.gate = _kinds(blocks, branches), gate
        znn._gate_number(gate)       # refuses what is no gate function before anything is made
        self.extents, self.device = tuple(extents), device
        self.params = {k: torch.from_numpy(np.ascontiguousarray(v)).to(device) for k, v in params.items()}
        self.random = znn.random_state(seed, device)
        plan = lambda f, fo: znn.Plan(f, fo, self.extents, ONES, mode)  # noqa: E731
        up = lambda kind: None if kind == "gated" else plan(maps, 4 * hidden if kind in LINES else hidden)  # noqa: E731
        self.plans = [(up(kind), plan(2 * hidden if kind in LINES else hidden, maps)) for kind in self.kinds]
        self.last = plan(maps, out_maps)

    def _branch(self, i, y, keep):
        """(result, what its backward pass reads beside that and y)"""
        kind, w1, b1 = self.kinds[i - 1], self.params["w1_%d" % i], self.params.get("b1_%d" % i)
        if kind == "gated":
            return znn.gated_fwd(y, w1, b1, self.gate, 0, keep)
        a = self.plans[i - 1][0].fwd(y, w1)
        if kind == "plain":
            return znn.transfer_fwd(a, b1, self.fn), None
        (z0, x0, z1, x1), dim = a.chunk(4), LINES[kind]
        h = a.new_empty((a.shape[0] // 2,) + a.shape[1:])
        znn.recurrence_fwd(z0, x0, None, dim, False, out=h.chunk(2)[0])
        znn.recurrence_fwd(z1, x1, None, dim, True, out=h.chunk(2)[1])
        return h, a

    def _branch_backward(self, i, gh, y, result, kept, grads):
        """The gradient of y; those of the branch's parameters go into ``grads``."""
        kind, w1, b1 = self.kinds[i - 1], "w1_%d" % i, "b1_%d" % i
        if kind == "gated":
            gy, grads[w1], grads[b1] = znn.gated_bwd(gh, y, self.params[w1], kept, self.gate)
            return gy
        up = self.plans[i - 1][0]
        if kind == "plain":
            ga = znn.transfer_bwd(gh, result, self.fn)
            grads[b1] = znn.bias_grad(ga)
        else:
            (z0, x0, z1, x1), (h0, h1), (g0, g1), dim = kept.chunk(4), result.chunk(2), gh.chunk(2), LINES[kind]
            ga = torch.empty_like(kept)
            gz0, gx0, gz1, gx1 = ga.chunk(4)
            znn.recurrence_bwd(g0, z0, x0, h0, None, dim, False, gz=gz0, gx=gx0)
            znn.recurrence_bwd(g1, z1, x1, h1, None, dim, True, gz=gz1, gx=gx1)
        grads[w1] = up.wgrad(y, ga)
        return up.bwd(ga, self.params[w1])

    def _forward(self, x, p, keep):
        """(out, what the backward pass reads): per block the norm's input, statistics and result, and what its branch made and kept."""
        q = self.params
        r = znn.dropout(x, p, self.random, 0) if p != 0 else x
        y, stats = znn.layernorm_fwd(r, q["norm_w_0"], q["norm_b_0"], self.eps, stats=keep)
        held = [(r, stats, y, None, None)]
        for i, (_, down) in enumerate(self.plans, 1):
            a, kept = self._branch(i, y, keep)
            h = down.fwd(a, q["w2_%d" % i])
            r, y, stats = znn.residual_norm_fwd(h, r, q["norm_w_%d" % i], q["norm_b_%d" % i], p, self.random, i, self.eps, stats=keep)
            if keep:
                held.append((r, stats, y, a, kept))
        return znn.transfer_fwd(self.last.fwd(y, q["w"]), q["b"], "logistic"), held

    def forward(self, x):
        """Prediction: nothing is dropped, and nothing kept for a backward pass."""
        return self._forward(x, 0.0, False)[0]

    def _backward(self, out, held, gout):
        q, grads = self.params, {}
        g = znn.transfer_bwd(gout, out, "logistic")
        grads["b"] = znn.bias_grad(g)
        grads["w"] = self.last.wgrad(held[-1][2], g)
        gy, gr = self.last.bwd(g, q["w"]), None     # gradients of y_i, and of r_i by what follows beside the norm
        for i in range(self.blocks, 0, -1):
            r, stats, _, a, kept = held[i]
            down = self.plans[i - 1][1]
            gr, gh, grads["norm_w_%d" % i], grads["norm_b_%d" % i] = znn.residual_norm_bwd(
                gy, gr, r, q["norm_w_%d" % i], stats, self.p, self.random, i)
            grads["w2_%d" % i] = down.wgrad(a, gh)
            gy = self._branch_backward(i, down.bwd(gh, q["w2_%d" % i]), held[i - 1][2], a, kept, grads)
        # no gradient reaches x: the sum of the branch and the first norm is wanted for the norm's parameters alone
        r, stats = held[0][:2]
        _, grads["norm_w_0"], grads["norm_b_0"] = znn.layernorm_bwd(gy, r, q["norm_w_0"], stats)
        return grads

    def train_round(self, x, target, eta, loss="cross_entropy"):
        """Forward, loss gradient, backward, update; returns (out, gradients)."""
        out, held = self._forward(x, self.p, True)
        grads = self._backward(out, held, znn.loss_grad(out, target, loss))
        for k, g in grads.items():
            znn.sgd_update(self.params[k], g, eta)
        znn.random_advance(self.random)
        return out, grads

    def capture_round(self, x, target, eta, loss="cross_entropy"):
        """Records one training round into a HIP graph and returns ``(replay, (out, gradients))``; see ``Net.capture_round``.
        Every replay drops other elements."""
        kept = {k: v.clone() for k, v in {**self.params, "": self.random}.items()}
        side = torch.cuda.Stream(device=self.device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):       # plans grow their workspaces outside the graph
            self.train_round(x, target, eta, loss)
            for k, v in kept.items():
                (self.params[k] if k else self.random).copy_(v)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outputs = self.train_round(x, target, eta, loss)
        return graph.replay, outputs
