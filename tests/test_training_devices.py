"""CPU: a context's calls run on its own device, so the plumbing for training programs refuses tensors of another one."""
from types import SimpleNamespace

import pytest
import torch

from paper_2308_14352_b200 import binding as B
from paper_2308_14352_b200 import training


@pytest.fixture
def contexts(monkeypatch):
    """Contexts on the devices 0 and 1, as emoe_create notes them; no call reaches them."""
    def create(device, nbytes, status):
        return 0x1000 * (device + 1)

    monkeypatch.setattr(B, "lib", lambda: SimpleNamespace(emoe_create=create, emoe_destroy=lambda ctx: 0))
    ctxs = [B.emoe_create(d, 0) for d in (0, 1)]
    yield ctxs
    for c in ctxs:
        B.emoe_destroy(c)


def _on(device, *shape, dtype=torch.float32):
    """What a tensor on a GPU shows of itself."""
    return SimpleNamespace(device=torch.device("cuda", device), shape=torch.Size(shape), dtype=dtype, dim=lambda: len(shape), is_contiguous=lambda: True)


def test_the_plumbing_keeps_to_the_contexts_device(contexts):
    for d in (0, 1):
        other = contexts[1 - d]
        assert training.ExpertRows(contexts[d], 64, 4, 2, device=d).device.index == d
        assert training.LowRankAdapters(contexts[d], _on(d, 2, 8, 64), _on(d, 2, 16, 8)).device.index == d
        with pytest.raises(ValueError, match="context"):
            training.ExpertRows(other, 64, 4, 2, device=d)
        with pytest.raises(ValueError, match="context"):
            training.LowRankAdapters(other, _on(d, 2, 8, 64), _on(d, 2, 16, 8))
        with pytest.raises(ValueError, match="context"):
            training.gate_backward(other, _on(d, 3, 8), _on(d, 3, 2, dtype=torch.int32), _on(d, 3, 2), True)


def test_a_destroyed_context_is_forgotten(contexts):
    B.emoe_destroy(contexts[1])
    assert B.context_device(contexts[1]) is None and B.context_device(contexts[0]) == 0
    training.ExpertRows(contexts[1], 64, 4, 2, device=0)   # not known here: as with a handle from elsewhere
