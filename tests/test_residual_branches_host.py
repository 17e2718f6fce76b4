"""Branches of a residual net that do not fit are refused, and parameters are those that the branches take.  Without a GPU."""
import pytest

from paper_1510_06706_amd import residual


@pytest.mark.parametrize("blocks,branches", [(2, ("gated",)), (1, ("lines",)), (1, ("gated", "plain")), (0, ("plain",))])
def test_refused(blocks, branches):
    with pytest.raises(ValueError, match="branch"):
        residual.residual_params(4, 3, blocks, 1, 7, branches)


def test_parameters():
    kinds = ("plain", "gated", "lines_y")
    p = residual.residual_params(4, 3, 3, 1, 7, kinds)
    ones = (1, 1, 1)
    assert [p["w1_%d" % i].shape for i in (1, 2, 3)] == [(3, 4) + ones, (6, 4) + ones, (12, 4) + ones]
    assert [p["w2_%d" % i].shape for i in (1, 2, 3)] == [(4, 3) + ones, (4, 3) + ones, (4, 6) + ones]
    assert p["b1_1"].shape == (3,) and p["b1_2"].shape == (6,) and "b1_3" not in p
    plain = residual.residual_params(4, 3, 2, 1, 7)
    assert all((plain[k] == v).all() for k, v in residual.residual_params(4, 3, 2, 1, 7, ("plain",) * 2).items())
