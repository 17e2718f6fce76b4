"""Gradients of biases and weights over many positions whose terms are all alike, so that the roundings of a running sum all point one way:
what a sum may be off by follows from how many additions follow each other in it."""
import pytest
import torch

from oracle import gated
from paper_1510_06706_amd import binding as znn

pytestmark = pytest.mark.gpu

# additions one after another that a term of the biases' sums passes: eight in a step of 32 positions, 2^16 / 32 steps, two and up to 16 of shares in a workgroup's
# threads, and as many as there are shares
CHAIN = 8 + 2048 + 2 + 16


# few features in, many out: few shares of many positions each; maps and rows whose gradients are stored
@pytest.mark.parametrize("axis,f,fo,n", [(1, 4, 4096, 1 << 20), (0, 4, 4096, 1 << 20), (0, 65, 2100, 1 << 21), (1, 65, 8192, 1 << 19), (1, 4, 16, 1 << 25)])
@pytest.mark.parametrize("term", [1.1, 0.9])
def test_biases_and_weights(axis, f, fo, n, term):
    print("case", axis, f, fo, n, term, flush=True)
    shape = lambda k: (n, k) if axis else (k, n)  # noqa: E731
    # gates of 1 with a slope of 1: du and dv are `term`
    kept = torch.ones(shape(2 * fo), device="cuda:0")
    gy = torch.full(shape(fo), term, device="cuda:0")
    x, w = torch.ones(shape(f), device="cuda:0"), torch.zeros(2 * fo, f, device="cuda:0")
    _, gw, gb = znn.gated_bwd(gy, x, w, kept, "rectify", axis, need_gx=False)
    want = n * float(gy.flatten()[0])
    shares = max(n >> 16, 129)
    off = float((gb.double() - want).abs().max()) / want / gated.HALF
    print("half-steps", off, flush=True)
    assert off <= CHAIN + shares / 16
    # by the bound that sums are documented to keep where their roundings point either way; a third of a chain's additions is what alike ones come to here
    assert off <= 24 + 2 * n ** 0.5
    assert float((gw.double() - want).abs().max()) / want / gated.HALF <= 24 + 2 * n ** 0.5
    del kept, gy, x
    torch.cuda.empty_cache()
