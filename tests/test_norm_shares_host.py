"""How far the sums of the parameters' gradients are cut up: from the workspace that a backward call asks for, without a GPU."""
import pytest

from paper_1510_06706_amd import binding as znn


def positions_of_a_share(rows, cols, axis):
    features, positions = (cols, rows) if axis else (rows, cols)
    shares = znn.layernorm_workspace_bytes(rows, cols, axis) // (8 * features)
    return positions / max(shares, 1)


@pytest.mark.parametrize("rows,cols,axis,most", [
    # by threads that take a position's features each: 64 to 1 rows of a workgroup at once, times 1024
    (1 << 28, 16, 1, 64 * 1024), ((1 << 27) + 1, 60, 1, 16 * 1024), (1 << 26, 128, 1, 16 * 1024), (16700001, 129, 1, 8 * 1024), (1 << 23, 1000, 1, 8 * 1024),
    (1 << 22, 2000, 1, 1024), (1 << 20, 16000, 1, 1024),
    # tiles of 256 to 32 columns, four additions a thread and tile, up to the columns that 32 bits of a tile's offsets reach
    (3, (1 << 28) - 100, 0, 64 * 1024), (24, (1 << 27) - 100, 0, 32 * 1024), (40, (1 << 26) - 61, 0, 16 * 1024), (120, (1 << 25) - 3, 0, 16 * 1024),
    (200, (1 << 24) - 100, 0, 8 * 1024), (500, (1 << 23) - 100, 0, 8 * 1024)])
def test_shares_of_the_largest_arrays(rows, cols, axis, most):
    """A thread adds up 1024 values before a share is left, whatever the array; the last tiles and rows may fall short."""
    assert positions_of_a_share(rows, cols, axis) <= most


@pytest.mark.parametrize("rows,cols,axis,shares", [(120, 96 ** 3, 0, 512), (40, 60 ** 3, 0, 1024), (5003, 1001, 1, 256), (16384, 512, 1, 512), (60000, 24, 1, 1024)])
def test_shares_of_ordinary_arrays(rows, cols, axis, shares):
    """What a chip holds at once: more would be read for nothing."""
    assert znn.layernorm_workspace_bytes(rows, cols, axis) == shares * 8 * (cols if axis else rows)


def test_workspaces_stay_small_beside_the_operands():
    for rows, cols, axis in ((1 << 28, 16, 1), (1 << 20, 20000, 1), (40, 1 << 28, 0), (600, 1 << 26, 0), (1 << 20, 16000, 1), (500, 1 << 25, 0)):
        assert znn.layernorm_workspace_bytes(rows, cols, axis) <= rows * cols * 4 / 100
    # extents that no memory holds
    for rows, cols, axis in (((1 << 32) - 1, 16384, 1), ((1 << 32) - 1, 1 << 26, 1), (1 << 26, 1 << 33, 0), (256, 1 << 34, 0)):
        assert znn.layernorm_workspace_bytes(rows, cols, axis) <= rows * cols * 4 / 100
