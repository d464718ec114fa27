"""GPU: every result of the low-rank calls as a whole (2-norms) against the formulas in 64 bits; the bounds and what they tell apart stand in
lowrank_precision.py."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.lowrank_precision import BF16, CASES, F32, Inputs

pytestmark = pytest.mark.gpu
CODE = {F32: B.DTYPE_F32, BF16: B.DTYPE_BF16}


def _run(c):
    desc = B.emoe_lowrank_desc(c.G, c.r, c.K, c.N, CODE[c.dtype], 0, 0, 0)
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(desc, c.n))
    new = lambda *s, dtype=F32: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    out = {"v": new(c.n, c.r), "y": new(c.n, c.N, dtype=c.dtype), "dx": new(c.n, c.K, dtype=c.dtype), "dA": new(c.G, c.r, c.K), "dB": new(c.G, c.N, c.r)}
    p = {k: t.data_ptr() for k, t in out.items()}
    vin = c.ref["v"].float()   # the formula's, so that dB shows its own sums' errors alone
    B.emoe_lowrank_forward(h, desc, c.A.data_ptr(), c.B.data_ptr(), c.scales.data_ptr(), c.x.data_ptr(), c.n, c.ids.data_ptr(), None, c.base.data_ptr(),
                           p["y"], p["v"])
    B.emoe_lowrank_backward(h, desc, c.A.data_ptr(), c.B.data_ptr(), c.scales.data_ptr(), c.x.data_ptr(), c.dy.data_ptr(), c.n, c.ids.data_ptr(), None,
                            vin.data_ptr(), c.dx_base.data_ptr(), p["dx"], p["dA"], p["dB"])
    torch.cuda.synchronize()
    assert B.emoe_device_status(h) == B.OK
    B.emoe_destroy(h)
    return out


@pytest.mark.parametrize("n,K,N,G,r,dtype,stream", CASES)
def test_results_as_a_whole(n, K, N, G, r, dtype, stream):
    c = Inputs(n, K, N, G, r, dtype, stream, device="cuda")
    if dtype == BF16:
        c.cancel()
    got, bounds = _run(c), c.bounds()
    for what, bound in bounds.items():
        if got[what].dtype == BF16:   # the result's rounding: half a step
            bound += torch.finfo(BF16).eps / 2 * c.ref[what].norm().item()
        err = (got[what].double() - c.ref[what]).norm().item()
        print(f"{what} {err:.3e} of {bound:.3e}, |ref| {c.ref[what].norm().item():.3e}")
        assert err <= bound, (what, err, bound)
