"""A residual net over the maps of every voxel, trained through the C ABI: what is put on the features of a
convolutional net to predict labels per voxel.

    r_0 = dropout(x),  y_0 = norm_0(r_0)
    r_i = r_(i-1) + dropout(W2_i f(W1_i y_(i-1) + b_i)),  y_i = norm_i(r_i)          i = 1 .. blocks
    out = logistic(W y_blocks + b)

The products are convolutions with 1 x 1 x 1 kernels; the end of every branch - dropout, node sum and the norm that the
next block begins with - is one library call in each direction.  Images keep their extents, so the net fits any volume.
This module only sequences library calls; every arithmetic step runs in libznn's kernels.
"""
from __future__ import annotations

import numpy as np

from . import binding as znn
from .synth import ONES, STREAM_BIAS, STREAM_KERNEL, uniform_pm1


def residual_params(maps, hidden, blocks, out_maps, seed):
    """Seeded fp32 parameters by name, in the distributions of ``synth.synthetic_params``."""
    p = {}

    def kernels(name, f, fo):
        p[name] = uniform_pm1(seed + 17 * len(p), STREAM_KERNEL, (fo, f) + ONES, float(np.sqrt(6.0 / f)))

    def small(name, n, around=0.0):
        p[name] = np.float32(around) + uniform_pm1(seed + 17 * len(p), STREAM_BIAS, (n,), 0.1)

    for i in range(blocks + 1):
        if i > 0:
            kernels("w1_%d" % i, maps, hidden)
            small("b1_%d" % i, hidden)
            kernels("w2_%d" % i, hidden, maps)
        small("norm_w_%d" % i, maps, 1.0)
        small("norm_b_%d" % i, maps)
    kernels("w", maps, out_maps)
    small("b", out_maps)
    return p


class ResidualNet:
    """``params`` as ``residual_params`` names them.  ``p`` is the probability to drop in training rounds; what is dropped
    follows from ``random``, the device's {seed, round}, which a round moves on by one."""

    def __init__(self, maps, hidden, blocks, out_maps, extents, params, p=0.1, fn="rectify", mode="auto", eps=znn.NORM_EPS, seed=0,
                 device="cuda:0"):
        import torch
        self.maps, self.blocks, self.p, self.fn, self.eps = maps, blocks, float(p), fn, eps
        self.extents, self.device = tuple(extents), device
        self.params = {k: torch.from_numpy(np.ascontiguousarray(v)).to(device) for k, v in params.items()}
        self.random = znn.random_state(seed, device)
        plan = lambda f, fo: znn.Plan(f, fo, self.extents, ONES, mode)  # noqa: E731
        self.plans = [(plan(maps, hidden), plan(hidden, maps)) for _ in range(blocks)]
        self.last = plan(maps, out_maps)

    def _forward(self, x, p, keep):
        """(out, what the backward pass reads): per block the norm's input, statistics and result, and both sides of f."""
        q = self.params
        r = znn.dropout(x, p, self.random, 0) if p != 0 else x
        y, stats = znn.layernorm_fwd(r, q["norm_w_0"], q["norm_b_0"], self.eps, stats=keep)
        held = [(r, stats, y, None)]
        for i, (up, down) in enumerate(self.plans, 1):
            a = znn.transfer_fwd(up.fwd(y, q["w1_%d" % i]), q["b1_%d" % i], self.fn)
            h = down.fwd(a, q["w2_%d" % i])
            r, y, stats = znn.residual_norm_fwd(h, r, q["norm_w_%d" % i], q["norm_b_%d" % i], p, self.random, i, self.eps, stats=keep)
            if keep:
                held.append((r, stats, y, a))
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
            r, stats, _, a = held[i]
            up, down = self.plans[i - 1]
            gr, gh, grads["norm_w_%d" % i], grads["norm_b_%d" % i] = znn.residual_norm_bwd(
                gy, gr, r, q["norm_w_%d" % i], stats, self.p, self.random, i)
            grads["w2_%d" % i] = down.wgrad(a, gh)
            ga = znn.transfer_bwd(down.bwd(gh, q["w2_%d" % i]), a, self.fn)
            grads["b1_%d" % i] = znn.bias_grad(ga)
            grads["w1_%d" % i] = up.wgrad(held[i - 1][2], ga)
            gy = up.bwd(ga, q["w1_%d" % i])
        # no gradient reaches x: the sum of the branch and the first norm is wanted for the norm's parameters alone
        r, stats, _, _ = held[0]
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
        import torch
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
