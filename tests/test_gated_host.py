"""What the gated unit and the gated recurrence refuse: on the host, before anything is launched, so without a GPU."""
import ctypes

import pytest
import torch

from paper_1510_06706_amd import binding as znn

P = ctypes.c_void_p(1 << 20)        # never dereferenced: every call here is refused
WS = 1 << 60


def call(name, **change):
    """The call with arguments that would do, but for the changes."""
    forms = {
        "gated_fwd": dict(fn=3, fan_in=4, fan_out=3, positions=5, axis=0, x=P, w=P, b=P, y=P, kept=None, ws=P, ws_bytes=WS, stream=None),
        "gated_bwd": dict(fn=3, fan_in=4, fan_out=3, positions=5, axis=1, gy=P, x=P, w=P, kept=P, gx=P, gw=P, gb=P, ws=P, ws_bytes=WS, stream=None),
        "recurrence_fwd": dict(outer=2, length=3, inner=4, reverse=0, z=P, x=P, h0=P, h=P, ws=P, ws_bytes=WS, stream=None),
        "recurrence_bwd": dict(outer=2, length=3, inner=4, reverse=1, gh=P, z=P, x=P, h=P, h0=P, gz=P, gx=P, gh0=P, ws=P, ws_bytes=WS, stream=None),
    }
    args = forms[name]
    assert set(change) <= set(args)
    return getattr(znn.lib(), "znn_" + name)(*{**args, **change}.values())


@pytest.mark.parametrize("name,pointers", [("gated_fwd", ["x", "w", "y"]), ("gated_bwd", ["gy", "x", "w", "kept", "gw"]),
                                           ("recurrence_fwd", ["z", "x", "h"]), ("recurrence_bwd", ["gh", "z", "x", "h", "gz", "gx"])])
def test_missing_operands(name, pointers):
    for p in pointers:
        assert call(name, **{p: None}) == znn.ZNN_EINVAL, p
        assert znn.last_error()


@pytest.mark.parametrize("name", ["gated_fwd", "gated_bwd"])
def test_gated_extents(name):
    for e in ("fan_in", "fan_out", "positions"):
        for v in (0, -1):
            assert call(name, **{e: v}) == znn.ZNN_EINVAL
    for axis in (-1, 2):
        assert call(name, axis=axis) == znn.ZNN_EINVAL
    for fn in (-1, 5):
        assert call(name, fn=fn) == znn.ZNN_EINVAL
    assert call(name, fan_in=1 << 10, positions=(1 << 28) + 1) == znn.ZNN_EUNSUPPORTED
    assert call(name, fan_out=1 << 10, positions=(1 << 28) + 1) == znn.ZNN_EUNSUPPORTED
    for e, v in (("fan_in", (1 << 20) + 1), ("fan_out", (1 << 20) + 1), ("positions", 1 << 31)):
        assert call(name, **{e: v}) == znn.ZNN_EUNSUPPORTED


@pytest.mark.parametrize("name", ["recurrence_fwd", "recurrence_bwd"])
def test_line_extents(name):
    for e in ("outer", "length", "inner"):
        for v in (0, -1):
            assert call(name, **{e: v}) == znn.ZNN_EINVAL
        assert call(name, **{e: (1 << 34) + 1}) == znn.ZNN_EUNSUPPORTED
    assert call(name, outer=1 << 19, length=1 << 19, inner=2) == znn.ZNN_EUNSUPPORTED


def need_of(name, shape):
    if name.startswith("gated"):
        return znn.gated_workspace_bytes(*shape, axis=0, which=znn.ZNN_PASS_BWD if name == "gated_bwd" else znn.ZNN_PASS_FWD)
    return znn.recurrence_workspace_bytes(*shape)


@pytest.mark.parametrize("name,shapes", [("gated_bwd", [(1, 1, 1), (40, 80, 1728), (200, 1000, 30000)]), ("recurrence_fwd", [(1, 1 << 20, 1), (1, 1 << 16, 512)]),
                                         ("recurrence_bwd", [(1, 1 << 20, 1), (1, 1 << 16, 512)])])
def test_workspace(name, shapes):
    extents = ("fan_in", "fan_out", "positions") if name.startswith("gated") else ("outer", "length", "inner")
    for shape in shapes:
        need = need_of(name, shape)
        change = dict(zip(extents, shape))
        if name.startswith("gated"):
            change["axis"] = 0
        if not need:
            continue
        assert call(name, ws=None, **change) == znn.ZNN_EWORKSPACE
        assert call(name, ws_bytes=need - 1, **change) == znn.ZNN_EWORKSPACE
        assert call(name, ws=ctypes.c_void_p((1 << 20) + 128), ws_bytes=need, **change) == znn.ZNN_EWORKSPACE


def test_workspace_queries():
    b = ctypes.c_size_t(0)
    L = znn.lib()
    assert L.znn_gated_workspace_bytes(4, 3, 5, 0, znn.ZNN_PASS_FWD, None) == znn.ZNN_EINVAL
    for which in (-1, znn.ZNN_PASS_WGRAD, 3):
        assert L.znn_gated_workspace_bytes(4, 3, 5, 0, which, ctypes.byref(b)) == znn.ZNN_EINVAL
    assert L.znn_gated_workspace_bytes(0, 3, 5, 0, 0, ctypes.byref(b)) == znn.ZNN_EINVAL
    assert L.znn_recurrence_workspace_bytes(1, 2, 3, None) == znn.ZNN_EINVAL
    assert L.znn_recurrence_workspace_bytes(1, 0, 3, ctypes.byref(b)) == znn.ZNN_EINVAL


X, W, B = torch.zeros(4, 5), torch.zeros(6, 4), torch.zeros(6)


@pytest.mark.parametrize("refused,match", [
    (lambda: znn.gated_fwd(X, W, B, "softplus"), "gate function"), (lambda: znn.gated_fwd(X, W, B, axis=2), "axis"),
    (lambda: znn.gated_fwd(X, torch.zeros(5, 4)), "weights"), (lambda: znn.gated_fwd(X, torch.zeros(6, 5)), "weights"),
    (lambda: znn.gated_fwd(X, torch.zeros(6, 4, 3)), "weights"), (lambda: znn.gated_fwd(X, W, axis=1), "weights"),
    (lambda: znn.gated_fwd(torch.zeros(4, 0), W), "array"), (lambda: znn.gated_fwd(X, W, torch.zeros(3)), "biases"),
    (lambda: znn.gated_bwd(X, X, W, torch.zeros(6, 5)), "gradient"), (lambda: znn.gated_bwd(torch.zeros(3, 5), X, W, torch.zeros(3, 5)), "kept"),
    (lambda: znn.gated_fwd(X, W, B), "GPU"), (lambda: znn.gated_bwd(torch.zeros(3, 5), X, W, torch.zeros(6, 5)), "GPU")])
def test_gated_arguments(refused, match):
    with pytest.raises(ValueError, match=match):
        refused()


@pytest.mark.parametrize("refused,match", [
    (lambda: znn.recurrence_fwd(X, X, dim=2), "dimension"), (lambda: znn.recurrence_fwd(X, X, dim=-3), "dimension"),
    (lambda: znn.recurrence_fwd(torch.zeros(()), torch.zeros(())), "dimension"), (lambda: znn.recurrence_fwd(torch.zeros(4, 0), torch.zeros(4, 0)), "lines"),
    (lambda: znn.recurrence_fwd(X, torch.zeros(4, 6)), "shape"), (lambda: znn.recurrence_fwd(X, X, torch.zeros(5)), "state"),
    (lambda: znn.recurrence_fwd(X, X, out=torch.zeros(5, 4)), "shape"), (lambda: znn.recurrence_bwd(X, X, X, torch.zeros(5, 4)), "shape"),
    (lambda: znn.recurrence_bwd(X, X, X, X, torch.zeros(4), dim=0), "state"), (lambda: znn.recurrence_fwd(X, X), "GPU"),
    (lambda: znn.recurrence_bwd(X, X, X, X), "GPU")])
def test_line_arguments(refused, match):
    with pytest.raises(ValueError, match=match):
        refused()


# lines are cut into pieces that are worked on side by side: nothing may be written over what another piece reads
STATES, ROWS = torch.zeros(40), torch.zeros(9, 5)


@pytest.mark.parametrize("refused", [
    lambda: znn.recurrence_fwd(X, X, out=X), lambda: znn.recurrence_fwd(ROWS[:4], torch.zeros(4, 5), out=ROWS[3:7]),
    lambda: znn.recurrence_fwd(X, X, STATES[:4], out=STATES[2:22].view(4, 5)), lambda: znn.recurrence_bwd(X, X, X, X, gz=X),
    lambda: znn.recurrence_bwd(X, X, X, X, gx=X), lambda: znn.recurrence_bwd(X, X, X, X, gz=ROWS[:4], gx=ROWS[3:7]),
    lambda: znn.recurrence_bwd(X, X, X, ROWS[:4], gx=ROWS[1:5])])
def test_results_that_share_memory_are_refused(refused):
    with pytest.raises(ValueError, match="memory of its own"):
        refused()


def test_results_side_by_side_are_not():
    a, b = ROWS[:4], ROWS[4:8]
    with pytest.raises(ValueError, match="GPU"):        # as far as that
        znn.recurrence_fwd(X, X, out=a)
    with pytest.raises(ValueError, match="GPU"):
        znn.recurrence_bwd(X, X, X, X, gz=a, gx=b)
