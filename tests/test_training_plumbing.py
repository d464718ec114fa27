"""CPU: what the plumbing for training programs refuses before any address reaches the library."""
import pytest
import torch

from paper_2308_14352_b200 import training

CTX = 0  # no call gets as far as the context


def test_tensors_off_the_gpu_are_refused():
    logits, ids, dg = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    with pytest.raises(ValueError):
        training.gate_backward(CTX, logits, ids, dg, True)
    with pytest.raises(ValueError):
        training.LowRankAdapters(CTX, torch.zeros(2, 8, 64), torch.zeros(2, 16, 8))
    er = training.ExpertRows(CTX, 64, 4, 2)
    with pytest.raises(ValueError):
        er.dispatch(torch.zeros(3, 64, dtype=torch.bfloat16), ids)


def test_rows_need_an_order():
    """An order that was never set, or whose setting was refused, is none."""
    er = training.ExpertRows(CTX, 64, 4, 2)
    rows, tokens = torch.zeros(0, 64, dtype=torch.bfloat16), torch.zeros(3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        er.dispatch(tokens, torch.zeros(3, 2, dtype=torch.int32))
    assert er.tokens == 0
    for call in (lambda: er.combine(rows), lambda: er.dispatch_backward(rows), lambda: er.combine_backward(rows)):
        with pytest.raises(ValueError):
            call()


def test_wrong_ranks_of_tensors_are_refused():
    with pytest.raises(ValueError):
        training.gate_backward(CTX, torch.zeros(8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), False)
    with pytest.raises(ValueError):
        training.gate_backward(CTX, torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3), False)
    with pytest.raises(ValueError):
        training.LowRankAdapters(CTX, torch.zeros(8, 64), torch.zeros(16, 8))


def test_the_gate_gradient_refuses_tokens_beyond_its_indices():
    from paper_2308_14352_b200 import binding as B

    call = lambda T: B.lib().emoe_gate_backward(None, 0x1000, T, 1, 0x2000, 0x3000, 1, B.GATE_SOFTMAX, 0x4000, None)  # noqa: E731
    assert call((1 << 31) - 1) == B.ERR_UNSUPPORTED and call(1 << 29) == B.ERR_UNSUPPORTED
    assert call((1 << 29) - 1) == B.ERR_INVALID_ARG  # all else in order: the context is missing
