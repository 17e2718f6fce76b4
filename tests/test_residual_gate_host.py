"""What a residual net's gated branches are gated by is checked when the net is made, not by its first pass.  Without a GPU."""
import pytest

from paper_1510_06706_amd import residual


@pytest.mark.parametrize("branches", [("gated", "plain"), ("plain", "lines_x"), None])
def test_gate_functions(branches):
    with pytest.raises(ValueError, match="gate function"):
        residual.ResidualNet(4, 3, 2, 1, (2, 2, 2), residual.residual_params(4, 3, 2, 1, 7, branches), branches=branches, gate="softplus", device="cpu")
