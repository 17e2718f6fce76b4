"""Arguments of the norm and dropout calls that Python hands on: what does not fit is refused, not cut off.  Without a GPU."""
import pytest
import torch

from paper_1510_06706_amd import binding as znn

X, V = torch.zeros(2, 3), torch.ones(2)
STATS = torch.zeros(2, 3)
CALLS = [lambda site: znn.dropout(X, 0.5, None, site), lambda site: znn.residual_norm_fwd(X, X, V, V, 0.5, None, site),
         lambda site: znn.residual_norm_bwd(X, None, X, V, STATS, 0.5, None, site)]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("site", [-1, 1 << 32, (1 << 32) + 5])
def test_sites_have_32_bits(call, site):
    with pytest.raises(ValueError, match="site"):
        call(site)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("site", [0, (1 << 32) - 1])
def test_sites_that_fit(call, site):
    """What is refused then are operands that are not on a GPU."""
    with pytest.raises(ValueError, match="cuda|CUDA|GPU"):
        call(site)
