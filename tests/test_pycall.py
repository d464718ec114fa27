"""CPU: the training calls' callables (csrc/pycall.cpp) hand arguments on as ctypes does, and refuse what does not fit."""
import ctypes
import itertools
import sys

import pytest

from paper_2308_14352_b200 import binding as B

ROWS = B.emoe_dispatch_desc(64, 4, 2, B.DTYPE_BF16, B.DTYPE_F32, 0, 0, 0)
ADAPTERS = B.emoe_lowrank_desc(4, 16, 64, 32, B.DTYPE_BF16, 0, 0, 0)
NAMES = ("emoe_dispatch", "emoe_dispatch_backward", "emoe_combine", "emoe_combine_backward", "emoe_gate_backward", "emoe_lowrank_forward",
         "emoe_lowrank_backward")


def _arguments(name):
    """Arguments that are in order but for the missing context, on addresses that are never followed."""
    out = []
    for i, t in enumerate(getattr(B.lib(), name).argtypes):
        out.append({ctypes.c_void_p: 0x1000 * i, ctypes.c_int: 2}.get(t, ADAPTERS if "lowrank" in name else ROWS))
    out[0] = None
    if "lowrank" in name:
        out[8 if name.endswith("backward") else 7] = None   # ids; off is given
    if name == "emoe_gate_backward":
        out[7] = B.GATE_SOFTMAX
    return out


@pytest.mark.parametrize("name", NAMES)
def test_the_same_statuses_as_through_ctypes(name):
    fast, slow, good = getattr(B._calls(), name), getattr(B.lib(), name), _arguments(name)
    seen = {fast(*good)}
    assert seen == {slow(*good)} == {B.ERR_INVALID_ARG}
    for i, j in itertools.combinations(range(1, len(good)), 2):
        for values in itertools.product((None, 0, 1, 3, -1, -(1 << 31), (1 << 31) - 1, (1 << 63) + 5), repeat=2):
            a, fits = list(good), True
            for k, v in zip((i, j), values):
                t = slow.argtypes[k]
                fits &= t is ctypes.c_void_p or (t is ctypes.c_int and v is not None and abs(v) < 1 << 31) or \
                    (t not in (ctypes.c_void_p, ctypes.c_int) and v is None)
                a[k] = v
            if fits:
                status = fast(*a)
                assert status == slow(*a), (i, j, values)
                seen.add(status)
    assert len(seen) >= 2   # (alignment, unsupported values: every argument has reached its place)


def test_addresses_above_63_bits_and_each_place():
    """Every place of the longest call, told apart by its alignment: an odd address in place i alone decides the status."""
    fast, good = B._calls().emoe_lowrank_backward, _arguments("emoe_lowrank_backward")
    good = [v | (1 << 63) if isinstance(v, int) and v > 2 else v for v in good]
    assert fast(*good) == B.ERR_INVALID_ARG
    for i in (2, 3, 4, 5, 6, 9, 10, 11, 12, 13, 14):
        a = list(good)
        a[i] += 2
        assert fast(*a) == B.ERR_ALIGNMENT, i


def test_what_does_not_fit_is_refused():
    f, good = B._calls().emoe_combine, _arguments("emoe_combine")
    for bad in (good[:-1], good + [0]):
        with pytest.raises(TypeError):
            f(*bad)
    with pytest.raises(TypeError):
        f(*good, stream=0)
    for i, value, error in ((2, 1.5, TypeError), (2, "x", TypeError), (2, 1 << 64, OverflowError), (3, 1 << 31, OverflowError), (3, -(1 << 31) - 1, OverflowError),
                            (3, None, TypeError), (3, 2.0, TypeError), (1, 4096, TypeError), (1, ADAPTERS, TypeError), (1, b"short", TypeError)):
        a = list(good)
        a[i] = value
        with pytest.raises(error):
            f(*a)
    from paper_2308_14352_b200 import _pycall
    for args in ((4096, "pp", (), B), (4096, "psxpppppp", (4,), B), (4096, "pspppppp", (), B), (0, "pppppppp", (), B)):
        with pytest.raises(ValueError):
            _pycall.bind(*args)


def test_nothing_is_kept_from_a_call():
    f, good = B._calls().emoe_combine, _arguments("emoe_combine")
    desc = B.emoe_dispatch_desc(64, 4, 2, B.DTYPE_BF16, B.DTYPE_F32, 0, 0, 0)
    good[1], address = desc, (1 << 40) + 16
    good[2] = address
    counts = [sys.getrefcount(x) for x in (desc, address)]
    for _ in range(1000):
        f(*good)
        try:
            f(*good[:3], "x", *good[4:])
        except TypeError:
            pass
    assert [sys.getrefcount(x) for x in (desc, address)] == counts
