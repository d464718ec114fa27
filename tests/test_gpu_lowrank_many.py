"""GPU: the low-rank kernels for many bf16 rows where their tiles, accumulators and factors are shared by rows of several adapters: what is not
finite stays where it belongs, two contexts work at once, and a captured graph takes new ids."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.helpers import side_by_side
from tests.test_gpu_lowrank import BF16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 512 << 20)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


def _all(c, ctx, v=None):
    y, v_out = c.forward(ctx)
    dx, dA, dB = c.backward(ctx, v_out if v is None else v)
    torch.cuda.synchronize()
    assert B.emoe_device_status(ctx) == B.OK
    return y, v_out, dx, dA, dB


SIZES = [(4100, 2056, 4104, 16), (1400, 4104, 8200, 64), (3000, 2056, 6152, 33), (2560, 4096, 6144, 5)]


@pytest.mark.parametrize("kind", ["ids", "off"])
@pytest.mark.parametrize("n,K,N,r", SIZES)
def test_what_is_not_finite_reaches_nobody_else(ctx, n, K, N, r, kind):
    """Bad rows and factors of adapter 2, bad rows of nobody: all other results have the bits of a call without them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    ids = torch.randint(0, 6, (n,), generator=g, device="cuda")
    make = lambda: Case(n, K, N, 6, r, BF16, kind, none=0.15, ids=ids)  # noqa: E731
    clean = make()
    y0, v0, dx0, dA0, dB0 = _all(clean, ctx)
    vin = v0.clone()
    c = make()
    assert torch.equal(c.ids, clean.ids) and torch.equal(c.x, clean.x)
    bad, none = c.ids == 2, c.ids < 0
    c.A[2, 0], c.A[2, r - 1], c.B[2] = float("nan"), float("-inf"), float("inf")
    c.x[bad], c.dy[bad] = float("inf"), float("nan")
    c.x[none], c.dy[none] = float("nan"), float("inf")
    vin[bad], vin[none] = float("nan"), float("inf")
    y, v, dx, dA, dB = _all(c, ctx, vin)
    good = (c.ids >= 0) & ~bad
    for a, b in ((y, y0), (dx, dx0), (v, v0)):
        assert torch.equal(a[good], b[good])
        assert not torch.isfinite(a[bad]).any()
        if kind == "ids":
            assert torch.equal(a[none], b[none])
        else:
            assert torch.isnan(a[none]).all()            # as they were
    others = [a for a in range(6) if a != 2]
    assert torch.equal(dA[others], dA0[others]) and torch.equal(dB[others], dB0[others])
    assert not torch.isfinite(dA[2]).any() and not torch.isfinite(dB[2]).any()


def test_one_bad_row_of_an_adapter_reaches_its_own_results(ctx):
    """A row in the middle of a tile: its y and dx, its adapter's gradients, nothing else."""
    c = Case(4100, 2056, 4104, 3, 16, BF16)
    y0, v0, dx0, dA0, dB0 = _all(c, ctx)
    at = (c.ids == 1).nonzero()[77, 0].item()
    c.x[at, 2055], c.dy[at, 0] = float("nan"), float("nan")
    vin = v0.clone()
    y, v, dx, dA, dB = _all(c, ctx, vin)
    rest = torch.arange(c.n, device="cuda") != at
    for a, b in ((y, y0), (v, v0), (dx, dx0)):
        assert torch.equal(a[rest], b[rest]) and torch.isnan(a[at]).all()
    assert torch.equal(dA[[0, 2]], dA0[[0, 2]]) and torch.equal(dB[[0, 2]], dB0[[0, 2]])
    assert torch.isnan(dA[1]).all()                                           # dv of the row is NaN
    assert torch.isnan(dB[1, 0]).all() and torch.equal(dB[1, 1:], dB0[1, 1:])  # one channel of dy


def test_two_contexts_on_two_streams():
    cases = [Case(4100, 2056, 4104, 5, 16, BF16, seed=1), Case(1500, 4104, 8200, 9, 40, BF16, seed=2, none=0.1)]
    hs = [B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, c.n)) for c in cases]
    outs = [(c.out(), torch.empty(c.n, c.r, device="cuda"), c.inn(), torch.empty(c.G, c.r, c.K, device="cuda"),
             torch.empty(c.G, c.N, c.r, device="cuda")) for c in cases]
    torch.cuda.synchronize()

    def job(c, h, o):
        def work(stream):
            c.forward(h, y=o[0], v=o[1], stream=stream)
            c.backward(h, o[1], dx=o[2], dA=o[3], dB=o[4], stream=stream)
        return work

    side_by_side([job(c, h, o) for c, h, o in zip(cases, hs, outs)], 20)
    torch.cuda.synchronize()
    for c, h, o in zip(cases, hs, outs):
        for what, got in zip(("y", "v", "dx", "dA", "dB"), o):
            c.check(what, got)
        assert B.emoe_device_status(h) == B.OK
        B.emoe_destroy(h)


@pytest.mark.parametrize("n,K,N,r", [(4100, 2056, 4104, 16), (1400, 4104, 8200, 40)])
def test_captured_and_replayed_on_new_rows(ctx, n, K, N, r):
    """Forward and backward in one graph; adapters of the rows, and how many each has, change between replays."""
    c = Case(n, K, N, 8, r, BF16)
    side = torch.cuda.Stream()
    y, v, dx = c.out(), torch.empty(n, r, device="cuda"), c.inn()
    dA, dB = torch.empty(8, r, K, device="cuda"), torch.empty(8, N, r, device="cuda")

    def both():
        c.forward(ctx, y=y, v=v, stream=side.cuda_stream)
        c.backward(ctx, v, dx=dx, dA=dA, dB=dB, stream=side.cuda_stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for seed, skew, none in ((3, 0.0, 0.0), (4, 3.0, 0.3), (5, 1.0, 0.95)):
        o = Case(n, K, N, 8, r, BF16, seed=seed, skew=skew, none=none)
        for m in ("ids", "x", "dy", "base", "dx_base", "A", "B", "scales"):
            getattr(c, m).copy_(getattr(o, m))
        graph.replay()
        torch.cuda.synchronize()
        for what, got in (("v", v), ("y", y), ("dx", dx), ("dA", dA), ("dB", dB)):
            o.check(what, got)
    assert B.emoe_device_status(ctx) == B.OK
