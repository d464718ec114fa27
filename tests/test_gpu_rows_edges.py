"""GPU: calls of the row operators that their documentation allows and that are easily forgotten: rows overwritten by their gradient at every
width, more picks than experts, rows of more than a megabyte, tokens of nothing but dropped pairs beside others."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.test_gpu_dispatch import BF16, F32, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 0)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


@pytest.mark.parametrize("T,d,k,tok,row,more", [
    (300, 521, 2, BF16, BF16, {}), (300, 522, 1, F32, BF16, {}), (77, 8200, 8, BF16, F32, {}), (2000, 1024, 8, F32, F32, {}), (2000, 100, 3, BF16, BF16, {"bad": 0.2}),
    (5, 4096, 2, F32, BF16, {"pad": (8, 24)}), (900, 2051, 4, F32, F32, {"pad": (0, 3)})])
def test_rows_overwritten_by_their_gradient(ctx, T, d, k, tok, row, more):
    c = Case(T, d, 8, k, tok, row, **more)
    _, _, dg, out = c.check_back(ctx)
    rows, dg2 = c.rows(c.drows), torch.full_like(dg, float("nan"))
    before = rows.clone()
    B.emoe_combine_backward(ctx, c.desc, c.dy.data_ptr(), T, c.slots.data_ptr(), c.w.data_ptr(), rows.data_ptr(), rows.data_ptr(), dg2.data_ptr(), 0)
    torch.cuda.synchronize()
    assert torch.equal(rows[:c.owned], out[:c.owned]) and torch.equal(rows[c.owned:], before[c.owned:]) and torch.equal(dg, dg2)


@pytest.mark.parametrize("T,k,E", [(5, 8, 1), (600, 3, 2), (3000, 8, 3), (1024, 2, 1)])
def test_the_same_expert_picked_twice_by_a_token(ctx, T, k, E):
    c = Case(T, 72, E, k, BF16, BF16, skew=0.5)
    out = c.dispatch(ctx)
    torch.cuda.synchronize()
    c.check_dispatch(out)
    c.check_back(ctx)


@pytest.mark.parametrize("T", [1025, 40])
def test_rows_of_more_than_a_megabyte(ctx, T):
    c = Case(T, 270000, 4, 2, F32, BF16, weighted=False)
    out = c.dispatch(ctx)
    torch.cuda.synchronize()
    for s in range(0, c.owned, 97):
        assert torch.equal(out["rows"][s], c.x[c.token[s]].to(BF16))
    y = c.tokens()
    B.emoe_combine(ctx, c.desc, out["rows"].data_ptr(), T, out["slots"].data_ptr(), None, y.data_ptr(), 0)
    torch.cuda.synchronize()
    assert torch.equal(y, 2 * c.x.to(BF16).float())


@pytest.mark.parametrize("T", [40, 5000])
def test_tokens_without_an_expert_beside_others(ctx, T):
    c = Case(T, 264, 8, 2, BF16, F32)
    c.ids[::3] = -1
    out = c.dispatch(ctx)
    y, dx = c.tokens(), c.tokens()
    dw = torch.full((T, 2), float("nan"), device="cuda")
    B.emoe_combine(ctx, c.desc, out["rows"].data_ptr(), T, out["slots"].data_ptr(), None, y.data_ptr(), 0)
    B.emoe_dispatch_backward(ctx, c.desc, out["rows"].data_ptr(), T, out["slots"].data_ptr(), c.w.data_ptr(), c.x.data_ptr(), dx.data_ptr(), dw.data_ptr(), 0)
    torch.cuda.synchronize()
    none = torch.arange(T, device="cuda") % 3 == 0
    for t in (y, dx, dw):
        assert (t[none] == 0).all() and torch.isfinite(t).all() and (t[~none] != 0).any()
    assert (out["slots"].view(T, 2)[none] == -1).all() and out["counts"].sum().item() == 2 * int((~none).sum())
    assert B.emoe_device_status(ctx) == B.ERR_DEVICE_CHECK
