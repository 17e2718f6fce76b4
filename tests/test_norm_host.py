"""What dropout, layer norm and the residual join refuse: on the host, before anything is launched, so without a GPU."""
import ctypes

import pytest

from paper_1510_06706_amd import binding as znn

P = ctypes.c_void_p(1 << 20)        # never dereferenced: every call here is refused
NAN, INF = float("nan"), float("inf")


def call(name, **change):
    """The call with arguments that would do, but for the changes."""
    forms = {
        "random_advance": dict(state=P, stream=None),
        "dropout": dict(rows=2, cols=3, p=0.5, state=P, site=0, x=P, y=P, stream=None),
        "layernorm_fwd": dict(rows=2, cols=3, axis=0, eps=1e-5, x=P, w=P, b=P, y=P, stats=None, stream=None),
        "layernorm_bwd": dict(rows=2, cols=3, axis=1, gy=P, x=P, w=P, stats=P, gx=P, gw=P, gb=P, ws=P, ws_bytes=1 << 30, stream=None),
        "residual_norm_fwd": dict(rows=2, cols=3, axis=0, eps=1e-5, p=0.5, state=P, site=0, h=P, x=P, w=P, b=P, r=P, y=P, stats=P,
                                  stream=None),
        "residual_norm_bwd": dict(rows=2, cols=3, axis=1, p=0.5, state=P, site=0, gy=P, gr=None, r=P, w=P, stats=P, gx=P, gh=P, gw=P,
                                  gb=P, ws=P, ws_bytes=1 << 30, stream=None),
    }
    args = forms[name]
    assert set(change) <= set(args)
    return getattr(znn.lib(), "znn_" + name)(*{**args, **change}.values())


@pytest.mark.parametrize("name,pointers", [
    ("random_advance", ["state"]), ("dropout", ["state", "x", "y"]), ("layernorm_fwd", ["x", "w", "b", "y"]),
    ("layernorm_bwd", ["gy", "x", "w", "stats", "gx", "gw", "gb"]),
    ("residual_norm_fwd", ["state", "h", "x", "w", "b", "r", "y"]),
    ("residual_norm_bwd", ["state", "gy", "r", "w", "stats", "gx", "gh", "gw", "gb"])])
def test_missing_operands(name, pointers):
    for p in pointers:
        assert call(name, **{p: None}) == znn.ZNN_EINVAL, p
        assert znn.last_error()


@pytest.mark.parametrize("name", ["dropout", "layernorm_fwd", "layernorm_bwd", "residual_norm_fwd", "residual_norm_bwd"])
def test_extents(name):
    for rows, cols in ((0, 3), (2, 0), (-1, 3), (2, -5)):
        assert call(name, rows=rows, cols=cols) == znn.ZNN_EINVAL
    assert call(name, rows=1 << 32, cols=1) == znn.ZNN_EUNSUPPORTED
    assert call(name, rows=1, cols=(1 << 34) + 1) == znn.ZNN_EUNSUPPORTED
    assert call(name, rows=(1 << 32) - 1, cols=1 << 34) == znn.ZNN_EUNSUPPORTED


@pytest.mark.parametrize("name", ["layernorm_fwd", "layernorm_bwd", "residual_norm_fwd", "residual_norm_bwd"])
def test_axis_and_features(name):
    for axis in (-1, 2):
        assert call(name, axis=axis) == znn.ZNN_EINVAL
    assert call(name, axis=0, rows=(1 << 28) + 1, cols=1) == znn.ZNN_EUNSUPPORTED
    assert call(name, axis=1, rows=1, cols=(1 << 28) + 1) == znn.ZNN_EUNSUPPORTED


@pytest.mark.parametrize("name", ["layernorm_fwd", "residual_norm_fwd"])
def test_eps(name):
    for eps in (0.0, -1e-5, NAN, INF):
        assert call(name, eps=eps) == znn.ZNN_EINVAL


@pytest.mark.parametrize("name", ["dropout", "residual_norm_fwd", "residual_norm_bwd"])
def test_probability_and_state(name):
    for p in (-1e-9, 1.0 + 1e-9, NAN, INF, -INF):
        assert call(name, p=p) == znn.ZNN_EINVAL
    assert call(name, state=ctypes.c_void_p((1 << 20) + 4)) == znn.ZNN_EINVAL
    assert call("random_advance", state=ctypes.c_void_p((1 << 20) + 4)) == znn.ZNN_EINVAL


@pytest.mark.parametrize("name", ["layernorm_bwd", "residual_norm_bwd"])
@pytest.mark.parametrize("axis,rows,cols", [(0, 40, 300000), (1, 9000, 700)])
def test_workspace(name, axis, rows, cols):
    need = znn.layernorm_workspace_bytes(rows, cols, axis)
    assert need > 0
    shape = dict(axis=axis, rows=rows, cols=cols)
    assert call(name, ws=None, **shape) == znn.ZNN_EWORKSPACE
    assert call(name, ws_bytes=need - 1, **shape) == znn.ZNN_EWORKSPACE
    assert call(name, ws=ctypes.c_void_p((1 << 20) + 128), ws_bytes=need, **shape) == znn.ZNN_EWORKSPACE


def test_workspace_query():
    b = ctypes.c_size_t(0)
    f = znn.lib().znn_layernorm_workspace_bytes
    assert f(2, 3, 0, None) == znn.ZNN_EINVAL
    assert f(0, 3, 0, ctypes.byref(b)) == znn.ZNN_EINVAL
    assert f(2, 3, 2, ctypes.byref(b)) == znn.ZNN_EINVAL
    assert f(2, 3, 1, ctypes.byref(b)) == znn.ZNN_OK


def program_rc(*ops):
    """What a program of operations (kind, buffers, options of Program.add) is answered with; ten buffers."""
    from paper_1510_06706_amd import program as zp
    P = zp.Program("cuda:0")
    for _ in range(10):
        P.buffer("given", (4,))
    for kind, buf, how in ops:
        P.add(kind, buf, **how)
    try:
        P.build()
    except znn.ZnnError as e:
        return e.code
    return znn.ZNN_OK


def test_operations_of_programs():
    from paper_1510_06706_amd import program as zp
    how = dict(maps=2, n=(1, 2, 2))
    eps = dict(how, window=zp.eps_bits(1e-5))
    forward, backward, drop = (zp.NORM_FWD, (0, 1, 2, 3, 4), eps), (zp.NORM_BWD, (5, 0, 1, 4, 6, 7, 8), how), (zp.DROPOUT, (0, 9, 3), how)
    assert program_rc(forward, backward, drop, (zp.RANDOM_ADVANCE, (9,), {})) == znn.ZNN_OK
    assert program_rc((zp.NORM_FWD, (0, 1, 2, 3), eps)) == znn.ZNN_OK                        # without statistics
    assert program_rc((zp.NORM_FWD, (0, 1, 2), eps)) == znn.ZNN_EINVAL
    assert program_rc((zp.NORM_FWD, (0, 1, 2, 3, 4, 5), eps)) == znn.ZNN_EINVAL
    assert program_rc((zp.NORM_BWD, (5, 0, 1, 4, 6, 7), how)) == znn.ZNN_EINVAL
    assert program_rc((zp.DROPOUT, (0, 9), how)) == znn.ZNN_EINVAL
    assert program_rc((zp.RANDOM_ADVANCE, (), {})) == znn.ZNN_EINVAL
    for bad in (0.0, -1.0, NAN, INF):
        assert program_rc((zp.NORM_FWD, (0, 1, 2, 3, 4), dict(how, window=zp.eps_bits(bad)))) == znn.ZNN_EINVAL
    join = (0, 1, 9, 2, 3, 4, 5, 6)
    assert program_rc((zp.JOIN_FWD, join, eps)) == program_rc((zp.JOIN_FWD, join[:7], eps)) == znn.ZNN_OK      # without statistics
    assert program_rc((zp.JOIN_FWD, join[:6], eps)) == znn.ZNN_EINVAL
    assert program_rc((zp.JOIN_FWD, join, dict(how, window=zp.eps_bits(0.0)))) == znn.ZNN_EINVAL
    assert program_rc((zp.NORM_BWD, (5, 0, 1, 4, 6, 7, 8, 3), how)) == znn.ZNN_OK            # with a gradient to add
    # an update of another extent than the norm's gradient
    assert program_rc(backward, (zp.UPDATE, (7, 1), dict(n=(1, 1, 2)))) == znn.ZNN_OK
    assert program_rc(backward, (zp.UPDATE, (7, 1), dict(n=(1, 1, 3)))) == znn.ZNN_EINVAL
    assert program_rc((zp.JOIN_FWD + 1, (0,), {})) == znn.ZNN_EINVAL


@pytest.mark.parametrize("p,parts", [(0.0, 0), (0.5, -2 ** 31), (0.25, 2 ** 30), (1e-12, 0), (1 - 2.0 ** -32, -1)])
def test_parts_of_two_to_the_32(p, parts):
    from paper_1510_06706_amd import program as zp
    assert zp.drop_parts(p) == (0, 0, parts)


@pytest.mark.parametrize("p", [-1e-9, 1.0, 1 - 1e-12, NAN, INF])
def test_parts_of_two_to_the_32_that_are_none(p):
    from paper_1510_06706_amd import program as zp
    with pytest.raises(ValueError):
        zp.drop_parts(p)
