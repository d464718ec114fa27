"""GPU: offsets of the low-rank adapters that descend or leave the rows.  They are in device memory, so no call can refuse them; nothing
outside the tensors of the call is touched."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.test_gpu_lowrank import BF16, F32, Case

pytestmark = pytest.mark.gpu
GUARD = 4096
FILL = {BF16: -1.5, F32: -1.5}


class Guarded:
    """A tensor with as much in front of it and behind it as no call may touch."""

    def __init__(self, *shape, dtype):
        n = torch.Size(shape).numel()
        self.all = torch.full((n + 2 * GUARD,), FILL[dtype], dtype=dtype, device="cuda")
        self.t = self.all[GUARD:GUARD + n].view(*shape)

    def whole(self):
        return bool((self.all[:GUARD] == FILL[self.all.dtype]).all()) and bool((self.all[-GUARD:] == FILL[self.all.dtype]).all())


def _far(n, G):
    """Ends whose distance is no 32-bit number: - 2^31 - n / 4 would count as nearly 2^31 rows."""
    off = torch.linspace(0, n, G + 1).long()
    off[1], off[2], off[G] = (1 << 31) - 1, -(1 << 31), (1 << 31) - 1
    off[3], off[4] = n // 4, -(1 << 31)
    return off.to(torch.int32).cuda()


# few and many rows, each type; the last two take the streaming kernels
SIZES = [(5, 64, 48, 8, F32), (700, 64, 96, 8, BF16), (4096, 64, 64, 16, F32), (4096, 2048, 4096, 16, BF16), (2560, 512, 14336, 32, BF16)]


@pytest.mark.parametrize("n,K,N,r,dtype", SIZES)
def test_far_offsets_stay_inside(n, K, N, r, dtype):
    G = 8
    c = Case(n, K, N, G, r, dtype, "off")
    good, c.off = c.off, _far(n, G)
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, n))
    y, v, dx = Guarded(n, N, dtype=dtype), Guarded(n, r, dtype=F32), Guarded(n, K, dtype=dtype)
    dA, dB = Guarded(G, r, K, dtype=F32), Guarded(G, N, r, dtype=F32)
    vin = torch.zeros(n, r, device="cuda")
    for call in (lambda: c.forward(h, y=y.t, v=v.t), lambda: c.backward(h, vin, dx=dx.t, dA=dA.t, dB=dB.t),
                 lambda: c.backward(h, vin, dx=None, dx_base=None, dA=None, dB=dB.t)):
        call()
        torch.cuda.synchronize()
        assert all(g.whole() for g in (y, v, dx, dA, dB))
    B.emoe_device_status(h)
    # the context is as good as before
    c.off = good
    y, v = c.forward(h)
    torch.cuda.synchronize()
    c.check("y", y), c.check("v", v)
    assert B.emoe_device_status(h) == B.OK
    B.emoe_destroy(h)


@pytest.mark.parametrize("n,K,N,r,dtype", SIZES)
def test_empty_segments_and_gaps_at_the_ends_are_right(n, K, N, r, dtype):
    """Rows in front of the first offset and behind the last belong to nobody; equal offsets are adapters without rows."""
    c = Case(n, K, N, 4, r, dtype, "off")
    at = [n // 5, n // 5, n // 2, n // 2, n - n // 7]
    c.off = torch.tensor(at, dtype=torch.int32, device="cuda")
    c.ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for a in range(4):
        c.ids[at[a]:at[a + 1]] = a
    c.define()
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, n))
    y, v = c.forward(h)
    dx, dA, dB = c.backward(h, v)
    assert B.emoe_device_status(h) == B.OK
    rows = c.mine()
    for what, got in (("v", v), ("y", y), ("dx", dx)):
        c.check(what, got, rows)
        assert torch.isnan(got[~rows]).all()
    c.check("dA", dA), c.check("dB", dB)
    B.emoe_destroy(h)
