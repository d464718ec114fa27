"""CPU: the widest channels that the low-rank calls take, and what is refused beyond them, before any kernel."""
import pytest

from paper_2308_14352_b200 import binding as B

WIDEST = 32767 * 256   # blocks of 256 channels of dA and of dB stand side by side in one grid of at most 65535


def _status(in_dim, out_dim, dtype):
    """Of both calls on addresses that are never followed; all in order but for the missing context is ERR_INVALID_ARG."""
    d = B.emoe_lowrank_desc(2, 1, in_dim, out_dim, dtype, 0, 0, 0)
    at = [0x1000 * (i + 1) for i in range(12)]
    f = B.lib().emoe_lowrank_forward(None, d, at[0], at[1], None, at[2], 2, at[3], None, None, at[4], None, None)
    b = B.lib().emoe_lowrank_backward(None, d, at[0], at[1], None, at[2], at[3], 2, at[4], None, at[5], None, at[6], at[7], at[8], None)
    return f, b, B.emoe_lowrank_workspace_bytes(d, 2) > 0


@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_the_widest_channels(dtype):
    taken, refused = (B.ERR_INVALID_ARG, B.ERR_INVALID_ARG, True), (B.ERR_UNSUPPORTED, B.ERR_UNSUPPORTED, False)
    assert _status(WIDEST, WIDEST, dtype) == taken
    assert _status(WIDEST + 8, 8, dtype) == refused and _status(8, WIDEST + 8, dtype) == refused
