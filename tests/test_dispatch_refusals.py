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
