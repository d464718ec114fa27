"""CPU: the bounds by which the GPU's low-rank results are judged hold for the formulas with whole values and break where values or vectors are
cut to fewer bf16 parts than the kernels promise."""
import pytest
import torch

from tests.lowrank_precision import BF16, CASES, Inputs

FIRST = 64      # channels of the results
ADAPTERS = 3    # of the cases', with their rows: the bounds go by rows per adapter


@pytest.fixture(autouse=True)
def one_thread():
    """Many small products: threads that share them wait for one another."""
    before = torch.get_num_threads()
    torch.set_num_threads(1)
    yield
    torch.set_num_threads(before)


def _broken(c, got):
    bounds = c.bounds(FIRST)
    ref = c.results(first=FIRST)
    return {what for what, bound in bounds.items() if (got[what] - ref[what]).norm().item() > bound}


@pytest.mark.parametrize("n,K,N,G,r,dtype,stream", CASES)
def test_fewer_parts_break_the_bounds(n, K, N, G, r, dtype, stream):
    n, G = (n * ADAPTERS // G, ADAPTERS) if G > ADAPTERS else (n, G)
    c = Inputs(n, K, N, G, r, dtype, stream)
    cut = lambda parts: _broken(c, c.results(vectors=parts, values=None if dtype == BF16 else parts, first=FIRST))  # noqa: E731
    assert cut(3) == set()
    outer = {"dA", "dB"}
    if dtype == BF16:
        assert cut(1) >= outer
        # many rows: chains of 1024, and vectors of 512 channels, cut nearly as much themselves
        seen = {what for what, short in (("dA", c.most <= 256 and (N <= 264 or not stream[1])), ("dB", c.most <= 256 or not stream[1])) if short}
        assert cut(2) >= seen and (seen or G == 1)
        c.cancel()
        one, two = (_broken(c, c.results(vectors=parts, first=FIRST)) for parts in (1, 2))
        assert one >= {"y", "dx"} and not two & {"y", "dx"}
    else:
        assert cut(1) == cut(2) == {"v", "y", "dx"} | outer
