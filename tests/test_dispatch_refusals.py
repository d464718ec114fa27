"""What the row, gate and low-rank calls refuse, without a GPU: every check stands in front of the first CUDA call, and the
context is the last of them, so that the codes show with none."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2308_14352_b200 import build, binding

    build.build()
    return binding.lib()


def _desc(**kw):
    from paper_2308_14352_b200 import binding as B

    f = dict(d=64, n_experts=8, top_k=2, token_dtype=B.DTYPE_BF16, row_dtype=B.DTYPE_BF16, reserved=0, token_stride=0, row_stride=0)
    f.update(kw)
    return B.emoe_dispatch_desc(**f)


def _calls(lib, desc, T=4, base=0x1000):
    """The four calls on addresses that are never followed."""
    d = None if desc is None else ctypes.byref(desc)
    at = lambda i: base + 0x1000 * i  # noqa: E731
    return [lib.emoe_dispatch(None, d, at(0), T, at(1), at(2), at(3), at(4), at(5), at(6), at(7), None),
            lib.emoe_dispatch_backward(None, d, at(0), T, at(1), at(2), at(3), at(4), at(5), None),
            lib.emoe_combine(None, d, at(0), T, at(1), at(2), at(3), None),
            lib.emoe_combine_backward(None, d, at(0), T, at(1), at(2), at(3), at(4), at(5), None)]


def test_rows_calls_refuse_bad_descriptions(lib):
    from paper_2308_14352_b200 import binding as B

    assert set(_calls(lib, None)) == {B.ERR_INVALID_ARG}
    for kw in ({"d": 0}, {"d": -8}, {"n_experts": 0}, {"n_experts": 257}, {"top_k": 0}, {"top_k": 9}, {"token_stride": 63}, {"row_stride": 1},
               {"token_stride": -1}, {"row_stride": -64}):
        assert set(_calls(lib, _desc(**kw))) == {B.ERR_INVALID_ARG}, kw
    for T in (0, -1):
        assert set(_calls(lib, _desc(), T)) == {B.ERR_INVALID_ARG}
    for kw in ({"token_dtype": B.DTYPE_F16}, {"row_dtype": 7}, {"d": 1 << 30}):
        assert set(_calls(lib, _desc(**kw))) == {B.ERR_UNSUPPORTED}, kw
    assert set(_calls(lib, _desc(), 1 << 29)) == {B.ERR_UNSUPPORTED}
    assert set(_calls(lib, _desc(), base=0x1001)) == {B.ERR_ALIGNMENT}
    assert set(_calls(lib, _desc(token_dtype=B.DTYPE_F32, row_dtype=B.DTYPE_F32), base=0x1002)) == {B.ERR_ALIGNMENT}
    assert set(_calls(lib, _desc())) == {B.ERR_INVALID_ARG}  # all else in order: the context is missing


def test_rows_calls_refuse_missing_buffers(lib):
    from paper_2308_14352_b200 import binding as B

    d = ctypes.byref(_desc())
    odd = ctypes.byref(_desc(token_dtype=B.DTYPE_F16))
    full = [0x1000 * (i + 1) for i in range(8)]
    for i in (0, 1, 3, 4, 5, 6, 7):                       # weights (2) may be missing
        a = list(full)
        a[i] = None
        assert lib.emoe_dispatch(None, d, a[0], 4, *a[1:], None) == B.ERR_INVALID_ARG
    # with an address off its type's boundary the code would be another one: the buffers are looked at first
    assert lib.emoe_dispatch_backward(None, d, 0x1001, 4, 0x2000, None, None, 0x3000, 0x4000, None) == B.ERR_INVALID_ARG   # dweights without x
    assert lib.emoe_dispatch_backward(None, d, 0x1001, 4, 0x2000, None, None, 0x3000, None, None) == B.ERR_ALIGNMENT
    assert lib.emoe_combine_backward(None, d, 0x1001, 4, 0x2000, None, None, 0x3000, 0x4000, None) == B.ERR_INVALID_ARG    # dgates without rows
    assert lib.emoe_combine_backward(None, d, 0x1001, 4, 0x2000, None, None, 0x3000, None, None) == B.ERR_ALIGNMENT
    assert lib.emoe_combine(None, odd, 0x1000, 4, 0x2000, None, 0x3000, None) == B.ERR_UNSUPPORTED


def test_gate_gradient_refusals(lib):
    from paper_2308_14352_b200 import binding as B

    call = lambda z=0x1000, T=4, E=8, ids=0x2000, dg=0x3000, k=2, mode=B.GATE_SOFTMAX, dz=0x4000: lib.emoe_gate_backward(  # noqa: E731
        None, z, T, E, ids, dg, k, mode, dz, None)
    for kw in ({"z": None}, {"ids": None}, {"dg": None}, {"dz": None}, {"T": 0}, {"E": 0}, {"E": 257}, {"k": 0}, {"k": 9}, {"E": 1, "k": 2}):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    assert call(mode=2) == B.ERR_UNSUPPORTED
    assert call(dz=0x4002) == B.ERR_ALIGNMENT and call(ids=0x2001) == B.ERR_ALIGNMENT
    assert call() == B.ERR_INVALID_ARG                    # the context is missing


def _lowrank(lib, desc, n=4, base=0x1000, **kw):
    """Forward and backward on addresses that are never followed; a keyword replaces one of them."""
    d = None if desc is None else ctypes.byref(desc)
    names = ("A", "B", "scales", "x", "dy", "ids", "v", "base", "y", "dA", "dB", "dx")
    p = {m: base + 0x1000 * i for i, m in enumerate(names)}
    p["off"] = None
    p.update(kw)
    f = lib.emoe_lowrank_forward(None, d, p["A"], p["B"], p["scales"], p["x"], n, p["ids"], p["off"], p["base"], p["y"], p["v"], None)
    b = lib.emoe_lowrank_backward(None, d, p["A"], p["B"], p["scales"], p["x"], p["dy"], n, p["ids"], p["off"], p["v"], p["base"], p["dx"], p["dA"],
                                  p["dB"], None)
    return f, b


def _ldesc(**kw):
    from paper_2308_14352_b200 import binding as B

    f = dict(n_adapters=4, rank=16, in_dim=64, out_dim=32, dtype=B.DTYPE_BF16, reserved=0, x_stride=0, y_stride=0)
    f.update(kw)
    return B.emoe_lowrank_desc(**f)


def test_lowrank_refusals(lib):
    from paper_2308_14352_b200 import binding as B

    both = lambda code: (code, code)  # noqa: E731
    assert _lowrank(lib, None) == both(B.ERR_INVALID_ARG)
    for kw in ({"n_adapters": 0}, {"n_adapters": 257}, {"rank": 0}, {"in_dim": 0}, {"out_dim": -8}, {"x_stride": 56}, {"y_stride": 24}, {"x_stride": -64}):
        assert _lowrank(lib, _ldesc(**kw)) == both(B.ERR_INVALID_ARG), kw
        assert B.emoe_lowrank_workspace_bytes(_ldesc(**kw), 4) == 0
    for kw in ({"dtype": B.DTYPE_F16}, {"dtype": 9}, {"rank": 65}, {"in_dim": 60}, {"out_dim": 12}, {"in_dim": 1 << 30}):
        assert _lowrank(lib, _ldesc(**kw)) == both(B.ERR_UNSUPPORTED), kw
    assert _lowrank(lib, _ldesc(), n=0) == both(B.ERR_INVALID_ARG)
    assert _lowrank(lib, _ldesc(), n=1 << 30) == both(B.ERR_UNSUPPORTED)
    assert _lowrank(lib, _ldesc(x_stride=68)) == both(B.ERR_ALIGNMENT)
    assert _lowrank(lib, _ldesc(y_stride=36)) == both(B.ERR_ALIGNMENT)
    assert _lowrank(lib, _ldesc(dtype=B.DTYPE_F32, x_stride=68))[0] == B.ERR_INVALID_ARG   # 16-byte rows: the context is missing
    assert _lowrank(lib, _ldesc(), base=0x1008) == both(B.ERR_ALIGNMENT)
    assert _lowrank(lib, _ldesc(), ids=None) == both(B.ERR_INVALID_ARG)
    assert _lowrank(lib, _ldesc(), off=0x9002, ids=None) == both(B.ERR_ALIGNMENT)
    # with an address off its boundary the code would be another one: what is missing is looked at first
    for missing in ("A", "B", "x", "y"):
        assert _lowrank(lib, _ldesc(), base=0x1008, **{missing: None})[0] == B.ERR_INVALID_ARG
    for missing in ("A", "B", "x", "dy", "v"):
        assert _lowrank(lib, _ldesc(), base=0x1008, **{missing: None})[1] == B.ERR_INVALID_ARG, missing
    assert _lowrank(lib, _ldesc(), base=0x1008, dx=None, dA=None, dB=None)[1] == B.ERR_INVALID_ARG
    assert _lowrank(lib, _ldesc(), base=0x1008, dx=None, dA=None, A=None, B=None, x=None)[1] == B.ERR_ALIGNMENT   # dB alone needs dy and v
    assert _lowrank(lib, _ldesc()) == both(B.ERR_INVALID_ARG)       # all else in order: the context is missing


def test_lowrank_workspace_grows_with_the_rows(lib):
    from paper_2308_14352_b200 import binding as B

    for d in (_ldesc(), _ldesc(n_adapters=256, rank=64, in_dim=8192, out_dim=8), _ldesc(dtype=B.DTYPE_F32, in_dim=14336, out_dim=4096)):
        sizes = [B.emoe_lowrank_workspace_bytes(d, n) for n in list(range(1, 700)) + [1000, 4096, 4097, 8192, 100000]]
        assert sizes[0] > 0 and sizes == sorted(sizes)
