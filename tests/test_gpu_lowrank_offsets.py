"""GPU: offsets of the low-rank adapters that descend or leave the rows.  They are in device memory, so no call can refuse them: one
of its kernels says so in the check word, and nothing outside the tensors of the call is touched."""
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


def _offsets(kind, n, G):
    off = torch.linspace(0, n, G + 1).long()
    if kind == "descends":
        off[G // 2] = off[G // 2 - 1] - 1
    elif kind == "overlaps":           # every other segment has all rows
        off[1::2], off[2::2] = n, 0
    elif kind == "beyond":
        off[G] = n + 1
    elif kind == "below":
        off[0] = -1
    elif kind == "far":
        # ends whose distance is no 32-bit number: - 2^31 - n / 4 would count as nearly 2^31 rows
        off[1], off[2], off[G] = (1 << 31) - 1, -(1 << 31), (1 << 31) - 1
        off[3], off[4] = n // 4, -(1 << 31)
    return off.to(torch.int32).cuda()


# few and many rows, each type; the last two take the streaming kernels, the very last one a way up whose runs are cut short
SIZES = [(5, 64, 48, 8, F32), (700, 64, 96, 8, BF16), (4096, 64, 64, 16, F32), (4096, 2048, 4096, 16, BF16), (2560, 512, 14336, 32, BF16)]


@pytest.mark.parametrize("kind", ["descends", "overlaps", "beyond", "below", "far"])
@pytest.mark.parametrize("n,K,N,r,dtype", SIZES)
def test_wrong_offsets_are_reported_and_stay_inside(n, K, N, r, dtype, kind):
    G = 8
    c = Case(n, K, N, G, r, dtype, "off")
    good, c.off = c.off, _offsets(kind, n, G)
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, n))
    y, v, dx = Guarded(n, N, dtype=dtype), Guarded(n, r, dtype=F32), Guarded(n, K, dtype=dtype)
    dA, dB = Guarded(G, r, K, dtype=F32), Guarded(G, N, r, dtype=F32)
    vin = torch.zeros(n, r, device="cuda")
    calls = {"forward": lambda: c.forward(h, y=y.t, v=v.t),
             "all": lambda: c.backward(h, vin, dx=dx.t, dA=dA.t, dB=dB.t),
             "dx": lambda: c.backward(h, None, dx=dx.t, dA=None, dB=None),
             "dA": lambda: c.backward(h, None, dx=None, dx_base=None, dA=dA.t, dB=None),
             "dB": lambda: c.backward(h, vin, dx=None, dx_base=None, dA=None, dB=dB.t)}
    said = {}
    for name, call in calls.items():
        call()
        said[name] = B.emoe_device_status(h)
        torch.cuda.synchronize()
        assert all(g.whole() for g in (y, v, dx, dA, dB)), name
    assert said == dict.fromkeys(calls, B.ERR_DEVICE_CHECK)
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
