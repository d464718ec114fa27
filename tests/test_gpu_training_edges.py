"""GPU: calls of the training operators that their documentation allows and that are easily forgotten: infinities beside a rank that fills
no tile, rows whose offsets pass 32 bits, a first call under capture, another stream than the default one."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.test_gpu_lowrank import BF16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 256 << 20)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


@pytest.mark.parametrize("n,K,rank", [(4, 64, 1), (4, 64, 5), (40, 64, 24), (700, 64, 40), (4100, 4104, 5), (2500, 4104, 40)])
def test_an_infinite_row_gives_infinities_at_every_rank(ctx, n, K, rank):
    """bf16, all factors and activations positive: the formula's results of row 1 are +inf, those of the others finite."""
    c = Case(n, K, K, 1, rank, BF16, scales=False)
    for t in (c.x, c.dy, c.A, c.B):
        t.copy_(t.abs() + 0.1)
    c.x[1, 5] = c.dy[1, 7] = float("inf")
    y, v = c.forward(ctx)
    dx, _, _ = c.backward(ctx, torch.ones(n, rank, device="cuda"), dA=None, dB=None)
    torch.cuda.synchronize()
    others = torch.arange(n, device="cuda") != 1
    for t in (v, y, dx):
        assert (t[1] == float("inf")).all() and torch.isfinite(t[others]).all()


# n, K, N, rank, values between rows: the last rows start beyond 2^31 values (and 4 GB); the fused kernels, the streaming ones
@pytest.mark.parametrize("n,K,N,rank,stride", [(36, 64, 64, 8, 1 << 26), (2200, 4096, 4096, 40, 1 << 20)])
def test_rows_whose_offsets_pass_32_bits(ctx, n, K, N, rank, stride):
    c = Case(n, K, N, 3, rank, BF16, none=0.1, pad=(stride - K, stride - N))
    y, v = c.forward(ctx)
    c.check("v", v)
    c.check("y", y)
    del y
    dx, dA, dB = c.backward(ctx, v)
    torch.cuda.synchronize()
    for what, got in (("dx", dx), ("dA", dA), ("dB", dB)):
        c.check(what, got)


FIRST_CALL = """
import sys
import torch
from paper_2308_14352_b200 import binding as B, training
from tests.test_gpu_lowrank import BF16, Case

kind, n = sys.argv[1], int(sys.argv[2])
torch.cuda.init()
ctx = B.emoe_create(0, 256 << 20)
g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
if kind == "adapters":
    c = Case(n, 2048, 4096, 4, 16, BF16)
    run = lambda: (lambda y, v: (y, v) + c.backward(ctx, v, stream=torch.cuda.current_stream().cuda_stream))(
        *c.forward(ctx, stream=torch.cuda.current_stream().cuda_stream))
else:
    x = torch.randn(n, 1024, device="cuda").bfloat16()
    ids = torch.randint(0, 8, (n, 2), device="cuda", dtype=torch.int32)
    logits, dg = torch.randn(n, 8, device="cuda"), torch.randn(n, 2, device="cuda")
    er = training.ExpertRows(ctx, 1024, 8, 2)
    def run():
        rows = er.dispatch(x, ids)
        y = er.combine(rows, dg)
        d_rows, d_gates = er.combine_backward(y, dg, rows)
        return rows, y, d_rows, d_gates, er.dispatch_backward(d_rows)[0], training.gate_backward(ctx, logits, ids, d_gates, True)
torch.cuda.synchronize()
with torch.cuda.graph(g, stream=s):
    captured = run()
g.replay()
g.replay()
torch.cuda.synchronize()
for a, b in zip(captured, run()):
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) and torch.isfinite(a).all()
B.emoe_destroy(ctx)
print("same bits")
"""


@pytest.mark.parametrize("kind,n", [("adapters", 24), ("adapters", 5000), ("rows", 16), ("rows", 3000)])
def test_a_programs_first_call_may_be_captured(kind, n):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL, kind, str(n)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same bits" in r.stdout, r.stderr[-2000:]


def test_calls_follow_the_stream_that_torch_works_on(ctx):
    """Inputs that a long chain on another stream makes just in front of the calls."""
    from paper_2308_14352_b200 import training

    n, d = 512, 512
    s = torch.cuda.Stream()
    ids = torch.randint(0, 4, (n, 1), device="cuda", dtype=torch.int32)
    A, Bm = torch.randn(4, 16, d, device="cuda"), torch.randn(4, d, 16, device="cuda")
    big = torch.randn(4096, 4096, device="cuda")
    er, ad = training.ExpertRows(ctx, d, 4, 1, torch.float32), training.LowRankAdapters(ctx, A, Bm)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        m = big
        for _ in range(20):
            m = torch.tanh(m @ big)
        x = m[:n, :d].contiguous()
        rows = er.dispatch(x, ids)
        out = ad.forward(rows, base=rows, off=er.off, keep=True)
        y = er.combine(out)
    torch.cuda.synchronize()
    e = ids[:, 0].long()
    want = x.double() + torch.einsum("nr,nor->no", torch.einsum("nd,nrd->nr", x.double(), A[e].double()), Bm[e].double())
    mag = x.double().abs() + torch.einsum("nr,nor->no", torch.einsum("nd,nrd->nr", x.double().abs(), A[e].double().abs()), Bm[e].double().abs())
    assert ((y.double() - want).abs() <= 2 * (d + 16 + 16) * 2.0 ** -24 * mag).all()
