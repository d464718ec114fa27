"""GPU: gradient of the gates where a token has no logit left (a padded batch's token): zeros, whatever the gradient of its gates holds."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 0)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


@pytest.mark.parametrize("mode", [B.GATE_SOFTMAX, B.GATE_SOFTMAX_RENORM])
@pytest.mark.parametrize("E,k", [(1, 1), (5, 2), (8, 8), (32, 2), (64, 4), (128, 8), (250, 3), (256, 8)])
def test_tokens_without_a_logit_get_zeros(ctx, E, k, mode):
    g = torch.Generator(device="cuda")
    g.manual_seed(E + k)
    T = 37
    z = torch.randn(T, E, generator=g, device="cuda")
    ids = torch.argsort(torch.rand(T, E, generator=g, device="cuda"), dim=1)[:, :k].to(torch.int32).contiguous()
    dg = torch.randn(T, k, generator=g, device="cuda")
    dead = torch.arange(T, device="cuda") % 3 == 1
    want = torch.empty_like(z)
    B.emoe_gate_backward(ctx, z.data_ptr(), T, E, ids.data_ptr(), dg.data_ptr(), k, mode, want.data_ptr())
    masked, bad = z.clone(), dg.clone()
    masked[dead] = float("-inf")
    for t, v in zip(dead.nonzero()[:, 0].tolist(), (float("inf"), float("-inf"), float("nan"), torch.finfo(torch.float32).max) * T):
        bad[t, t % k] = v
    got = torch.full_like(z, float("nan"))
    B.emoe_gate_backward(ctx, masked.data_ptr(), T, E, ids.data_ptr(), bad.data_ptr(), k, mode, got.data_ptr())
    torch.cuda.synchronize()
    assert (got[dead] == 0).all()
    assert torch.equal(got[~dead], want[~dead])


@pytest.mark.parametrize("E,k", [(8, 2), (128, 8)])
def test_renormalised_over_picks_without_a_logit(ctx, E, k):
    """The picks' logits alone are missing: the token's softmax over them has nothing, whatever the others hold."""
    z = torch.randn(6, E, device="cuda")
    z[2, :k] = float("-inf")
    ids = torch.arange(k, device="cuda", dtype=torch.int32).repeat(6, 1)
    dg = torch.randn(6, k, device="cuda")
    dg[2, 0] = float("nan")
    got = torch.full_like(z, float("nan"))
    B.emoe_gate_backward(ctx, z.data_ptr(), 6, E, ids.data_ptr(), dg.data_ptr(), k, B.GATE_SOFTMAX_RENORM, got.data_ptr())
    torch.cuda.synchronize()
    assert (got[2] == 0).all() and torch.isfinite(got).all()
