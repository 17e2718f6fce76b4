"""Results that share memory with an operand or with another result are refused at the C boundary, before anything is launched: without a GPU."""
import ctypes

import pytest

from paper_1510_06706_amd import binding as znn

MIB = 1 << 20
WS = 1 << 60

# (results, operands) with the elements that the calls below give each
FORMS = {
    "gated_fwd": (dict(y=15, kept=30), dict(x=20, w=24, b=6)),
    "gated_bwd": (dict(gx=20, gw=24, gb=6), dict(gy=15, x=20, w=24, kept=30)),
    "recurrence_fwd": (dict(h=24), dict(z=24, x=24, h0=8)),
    "recurrence_bwd": (dict(gz=24, gx=24, gh0=8), dict(gh=24, z=24, x=24, h=24, h0=8)),
}
ORDER = {
    "gated_fwd": ["x", "w", "b", "y", "kept"], "gated_bwd": ["gy", "x", "w", "kept", "gx", "gw", "gb"],
    "recurrence_fwd": ["z", "x", "h0", "h"], "recurrence_bwd": ["gh", "z", "x", "h", "h0", "gz", "gx", "gh0"],
}
EXTENTS = {"gated_fwd": (3, 4, 3, 5, 0), "gated_bwd": (3, 4, 3, 5, 1), "recurrence_fwd": (2, 3, 4, 0), "recurrence_bwd": (2, 3, 4, 1)}


def call(name, places):
    """Pointers a MiB apart, never read, but for those given; every call here is refused."""
    at = {k: (8 + i) * MIB for i, k in enumerate(ORDER[name])}
    at.update(places(at))
    return getattr(znn.lib(), "znn_" + name)(*EXTENTS[name], *(ctypes.c_void_p(at[k]) for k in ORDER[name]), ctypes.c_void_p(MIB), WS, None)


PAIRS = [(name, r, o) for name, (results, operands) in FORMS.items() for r in results for o in list(operands) + [k for k in results if k > r]]


@pytest.mark.parametrize("name,result,other", PAIRS)
def test_refused(name, result, other):
    sizes = {**FORMS[name][0], **FORMS[name][1]}
    # the same place, the other's last element, this one's last element
    for shift in (0, 4 * (sizes[other] - 1), -4 * (sizes[result] - 1)):
        assert call(name, lambda at: {result: at[other] + shift}) == znn.ZNN_EINVAL, shift
        assert b"share" in znn.last_error().encode()


def test_other_refusals_come_first():
    """A result over an operand hides no missing workspace."""
    L = znn.lib()
    need = znn.recurrence_workspace_bytes(1, 1 << 20, 1)
    assert need
    p = ctypes.c_void_p(8 * MIB)
    assert L.znn_recurrence_fwd(1, 1 << 20, 1, 0, p, p, None, p, None, 0, None) == znn.ZNN_EWORKSPACE
