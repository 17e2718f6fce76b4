"""Seeded parameters of nets that begin with a norm or a bias: their maps are those that the first convolution takes."""
import numpy as np
import pytest

from oracle import net as onet
from paper_1510_06706_amd import synth

LAYERS = [("layernorm",), ("transfer", "tanh"), ("dropout", 0.5), ("conv", 3, 4, (1, 2, 2)), ("layernorm", 1e-3), ("transfer", "logistic")]


def test_layers_before_the_first_convolution():
    params = synth.synthetic_params(LAYERS, 5)
    assert [None if p is None else {k: v.shape for k, v in p.items()} for p in params] == [
        {"w": (3,), "b": (3,)}, {"b": (3,)}, None, {"w": (4, 3, 1, 2, 2)}, {"w": (4,), "b": (4,)}, {"b": (4,)}]
    acts, _ = onet.forward(LAYERS, params, np.ones((3, 2, 4, 5)))
    assert acts[-1].shape == (4, 2, 3, 4)


def test_layers_behind_a_convolution_keep_theirs():
    """What seeds gave before: the last convolution's maps."""
    tail = [("conv", 1, 5, (3, 3, 3)), ("transfer",), ("layernorm",), ("conv", 5, 2, (1, 1, 1)), ("layernorm",), ("transfer",)]
    assert [len(p["b"]) for p in synth.synthetic_params(tail, 1) if "b" in p] == [5, 5, 2, 2]


def test_nets_without_convolutions_tell_no_maps():
    with pytest.raises(ValueError, match="convolution"):
        synth.synthetic_params([("layernorm",)], 1)
