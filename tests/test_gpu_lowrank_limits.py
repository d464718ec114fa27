"""GPU: low-rank adapters beside the widest projection that the calls take: the blocks of both outer products fill one grid."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.test_gpu_lowrank import F32, Case
from tests.test_lowrank_limits import WIDEST

pytestmark = pytest.mark.gpu


def test_the_widest_channels_on_both_sides():
    c = Case(2, WIDEST, WIDEST, 2, 1, F32, ids=torch.tensor([1, 0], device="cuda"), scales=False)
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, c.n))
    y, v = c.forward(h)
    dx, dA, dB = c.backward(h, v)
    torch.cuda.synchronize()
    for what, got in (("v", v), ("y", y), ("dx", dx), ("dA", dA), ("dB", dB)):
        c.check(what, got)
    assert B.emoe_device_status(h) == B.OK
    B.emoe_destroy(h)
