"""GPU parity: low-rank adapters (emoe_lowrank_forward / _backward) against the definition in 64 bits.

Tolerances.  A sum of n products in fp32, in whatever order, is off by at most (n + 1) 2^-24 of the sum of the magnitudes; the tensor
cores may cut instead of round when they add, which doubles that.  Splitting an fp32 value into three bf16 parts is exact, the left-out
products are below 3 * 2^-24 of a product.  In bf16 results the low-rank vector has two parts: 2^-16 of each of its values.  A
result is rounded once, by half a step of its type."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.helpers import side_by_side

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CODE = {F32: B.DTYPE_F32, BF16: B.DTYPE_BF16}
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 256 << 20)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


def _view(rows, d, dtype, pad, fill=None):
    v = torch.full((rows, d + pad), float("nan"), dtype=dtype, device="cuda")[:, :d]
    if fill is not None:
        v.copy_(fill)
    return v


def _ptr(t):
    return None if t is None else t.data_ptr()


class Case:
    def __init__(self, n, K, N, G, r, dtype, kind="ids", none=0.0, skew=0.0, scales=True, pad=(0, 0), seed=0, ids=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 31 * n + r)
        self.n, self.K, self.N, self.G, self.r, self.dtype, self.pad = n, K, N, G, r, dtype, pad
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        if ids is None:
            p = torch.arange(1, G + 1, device="cuda", dtype=F32) ** -skew
            ids = torch.multinomial(p, n, replacement=True, generator=g)
        self.ids = ids.to(torch.int32)
        if none:
            self.ids[torch.rand(n, generator=g, device="cuda") < none] = -1
        self.off = None
        if kind == "off":  # sorted, rows of no adapter behind the last
            key = torch.where(self.ids < 0, G, self.ids)
            self.ids = torch.sort(key).values.to(torch.int32)
            self.off = torch.searchsorted(self.ids, torch.arange(G + 1, device="cuda", dtype=torch.int32)).to(torch.int32)
            self.ids = torch.where(self.ids == G, -1, self.ids)
        self.A = (randn(G, r, K) * K ** -0.5).to(dtype)
        self.B = (randn(G, N, r) * 0.1).to(dtype)
        self.scales = torch.rand(G, generator=g, device="cuda") * 2 - 0.5 if scales else None
        self.x, self.dy = self.inn(randn(n, K)), self.out(randn(n, N))
        self.base, self.dx_base = self.out(randn(n, N)), self.inn(randn(n, K))
        self.desc = B.emoe_lowrank_desc(G, r, K, N, CODE[dtype], 0, K + pad[0] if pad[0] else 0, N + pad[1] if pad[1] else 0)
        self.define()

    def inn(self, fill=None):
        return _view(self.n, self.K, self.dtype, self.pad[0], fill)

    def out(self, fill=None):
        return _view(self.n, self.N, self.dtype, self.pad[1], fill)

    def define(self):
        """Results and sums of magnitudes in 64 bits, adapter by adapter."""
        n, K, N, G, r = self.n, self.K, self.N, self.G, self.r
        zero = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")  # noqa: E731
        self.ref = {"v": zero(n, r), "y": self.base.double().clone(), "dv": zero(n, r), "dx": self.dx_base.double().clone(),
                    "dA": zero(G, r, K), "dB": zero(G, N, r)}
        self.mag = {k: t.abs().clone() for k, t in self.ref.items()}
        self.rows_of = [(self.ids == a).nonzero()[:, 0] for a in range(G)]
        for a, at in enumerate(self.rows_of):
            A, Bm, x, dy = self.A[a].double(), self.B[a].double(), self.x[at].double(), self.dy[at].double()
            s = 1.0 if self.scales is None else self.scales[a].double()
            for out, f in ((self.ref, lambda t: t), (self.mag, torch.abs)):
                S = f(s) if torch.is_tensor(s) else s
                v, dv = f(x) @ f(A).t(), S * (f(dy) @ f(Bm))
                out["v"][at], out["dv"][at] = v, dv
                out["y"][at] += S * v @ f(Bm).t()
                out["dx"][at] += dv @ f(A)
                out["dA"][a] = dv.t() @ f(x)
                out["dB"][a] = S * (f(dy).t() @ v)

    def tolerance(self, what, dtype):
        """Roundings of the sums that lead to a result, largest number of rows of an adapter included; half a step of its type."""
        m = max([len(v) for v in self.rows_of] + [1])
        sums = {"v": self.K, "y": self.K + self.r, "dv": self.N, "dx": self.N + self.r, "dA": self.N + m, "dB": self.K + m}[what]
        parts = 2.0 ** -16 if dtype == BF16 and what in ("y", "dx") else 0.0
        return (2 * (sums + 16) * STEP + parts) * self.mag[what] + torch.finfo(dtype).eps / 2 * self.ref[what].abs() * (1 + 2.0 ** -8)

    def check(self, what, got, rows=None):
        ref, tol = self.ref[what], self.tolerance(what, got.dtype)
        if rows is not None:
            got, ref, tol = got[rows], ref[rows], tol[rows]
        assert torch.isfinite(got).all(), what
        worst = ((got.double() - ref).abs() - tol).max().item() if got.numel() else 0.0
        assert worst <= 1e-30, (what, worst, (got.double() - ref).abs().max().item())

    def which(self):
        return (None, self.off.data_ptr()) if self.off is not None else (self.ids.data_ptr(), None)

    def forward(self, ctx, y=None, base="own", v="new", stream=0):
        y = self.out() if y is None else y
        base = self.base if isinstance(base, str) else base
        v = torch.full((self.n, self.r), float("nan"), device="cuda") if isinstance(v, str) else v
        B.emoe_lowrank_forward(ctx, self.desc, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scales), self.x.data_ptr(), self.n, *self.which(),
                               _ptr(base), y.data_ptr(), _ptr(v), stream)
        return y, v

    def backward(self, ctx, v, dx="new", dx_base="own", dA="new", dB="new", stream=0):
        new = lambda t, *s: torch.full(s, float("nan"), device="cuda") if isinstance(t, str) else t  # noqa: E731
        dx = self.inn() if isinstance(dx, str) else dx
        dx_base = self.dx_base if isinstance(dx_base, str) else dx_base
        dA, dB = new(dA, self.G, self.r, self.K), new(dB, self.G, self.N, self.r)
        B.emoe_lowrank_backward(ctx, self.desc, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scales), self.x.data_ptr(), self.dy.data_ptr(), self.n,
                                *self.which(), _ptr(v), _ptr(dx_base), _ptr(dx), _ptr(dA), _ptr(dB), stream)
        return dx, dA, dB

    def mine(self):
        """Rows that a call writes: with offsets those of an adapter, with ids all."""
        return (self.ids >= 0) if self.off is not None else torch.ones_like(self.ids, dtype=torch.bool)


# n, K, N, adapters, rank, type, more
CASES = [
    (1, 64, 64, 1, 16, BF16, {}),
    (1, 4096, 4096, 4, 16, BF16, {}),
    (1, 8, 8, 1, 1, BF16, {}),                                         # the smallest of everything
    (1, 8, 16, 2, 3, F32, {"scales": False}),
    (24, 768, 1024, 16, 16, BF16, {"none": 0.2}),
    (24, 768, 1024, 16, 8, F32, {"none": 0.2}),
    (37, 1104, 776, 5, 12, BF16, {}),                                  # odd sizes: K and N no multiple of a warp's step
    (37, 1104, 776, 5, 12, F32, {"pad": (4, 12)}),
    (64, 520, 264, 64, 5, BF16, {}),                                   # odd rank: single values of a factor's row
    (65, 520, 264, 3, 20, BF16, {"pad": (8, 24)}),                     # ranks that are no whole words of the wider kernels
    (200, 136, 96, 2, 40, BF16, {}),
    (200, 136, 96, 2, 33, F32, {"none": 0.5}),
    (130, 256, 512, 1, 64, BF16, {}),
    (130, 256, 512, 1, 64, F32, {}),
    (512, 264, 136, 7, 24, BF16, {"skew": 1.1}),
    (513, 264, 136, 7, 24, BF16, {"skew": 1.1, "none": 0.1}),
    (1024, 264, 136, 7, 24, BF16, {"skew": 1.1}),                      # the last size whose rows every CTA looks up
    (1025, 264, 136, 7, 24, BF16, {"skew": 1.1, "none": 0.1}),         # the first that is sorted
    (1024, 136, 64, 256, 16, F32, {"none": 0.3}),
    (777, 72, 2056, 256, 4, BF16, {"none": 0.3}),                      # all adapters there can be, and rows of none
    (1500, 200, 88, 256, 16, F32, {}),
    (2100, 512, 512, 3, 32, BF16, {"skew": 2.0}),
    (2100, 136, 128, 3, 64, BF16, {"skew": 1.0}),
    (1030, 64, 72, 2, 48, F32, {}),
    (900, 384, 640, 8, 16, BF16, {"kind": "off"}),
    (900, 384, 640, 8, 16, F32, {"kind": "off", "none": 0.25}),
    (40, 384, 640, 8, 32, BF16, {"kind": "off", "none": 0.25}),
    (3000, 1024, 1032, 4, 16, BF16, {"kind": "off", "skew": 1.5}),     # several chunks of rows per adapter, and adapters with one
    (5, 128, 128, 200, 16, BF16, {"kind": "off"}),                     # most adapters without rows
    # bytes of the rows enough for the streaming kernels
    (4000, 2056, 4104, 5, 16, BF16, {"skew": 1.0}),                    # channels that end inside a tile, one value of them
    (4001, 2056, 4104, 256, 12, BF16, {"none": 0.4}),                  # short segments, several to a tile's rows, and a long one of none
    (2500, 4104, 6152, 3, 5, BF16, {"pad": (8, 24)}),                  # odd rank: vectors and factors by single values
    (9000, 1032, 2048, 1, 32, BF16, {}),                               # one adapter: every run is part of its rows
    (5000, 2048, 3080, 100, 20, BF16, {"kind": "off", "skew": 1.5, "none": 0.2}),
    (1300, 4096, 8200, 2, 64, BF16, {"kind": "off"}),
    (3000, 2056, 2056, 9, 40, BF16, {"none": 0.1, "skew": 2.0}),
    (2200, 2048, 3000, 200, 33, BF16, {}),
    (40000, 520, 264, 3, 16, BF16, {"skew": 1.0}),                     # more tiles than one round of runs holds
    (20000, 72, 520, 30, 64, BF16, {"kind": "off", "none": 0.01}),
]


@pytest.mark.parametrize("n,K,N,G,r,dtype,more", CASES)
def test_forward_and_backward(ctx, n, K, N, G, r, dtype, more):
    c = Case(n, K, N, G, r, dtype, **more)
    y, v = c.forward(ctx)
    dx, dA, dB = c.backward(ctx, v)
    torch.cuda.synchronize()
    rows = c.mine()
    c.check("v", v, rows)
    c.check("y", y, rows)
    c.check("dx", dx, rows)
    c.check("dA", dA)
    c.check("dB", dB)
    for t in (y, dx, v):
        assert torch.isnan(t[~rows]).all()                             # rows behind the last segment: as they were
    none = rows & (c.ids < 0)
    assert torch.equal(y[none], c.base[none]) and torch.equal(dx[none], c.dx_base[none]) and (v[none] == 0).all()
    assert B.emoe_device_status(ctx) == B.OK
    # the same bits again, in place and without what is not wanted
    y2 = c.out(c.base)
    c.forward(ctx, y=y2, base=y2, v=None)
    dx2 = c.inn(c.dx_base)
    c.backward(ctx, None, dx=dx2, dx_base=dx2, dA=None, dB=None)
    _, dA2, _ = c.backward(ctx, None, dx=None, dx_base=None, dB=None)
    _, _, dB2 = c.backward(ctx, v, dx=None, dx_base=None, dA=None)
    torch.cuda.synchronize()
    assert torch.equal(y2[rows], y[rows]) and torch.equal(dx2[rows], dx[rows])
    assert torch.equal(y2[~rows], c.base[~rows])
    assert torch.equal(dA2, dA) and torch.equal(dB2, dB)


@pytest.mark.parametrize("n", [3, 600])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_without_a_base(ctx, n, dtype):
    c = Case(n, 128, 96, 4, 16, dtype, none=0.3)
    c.base.zero_(); c.dx_base.zero_()
    c.define()
    y, v = c.forward(ctx, base=None)
    dx, _, _ = c.backward(ctx, v, dx_base=None)
    torch.cuda.synchronize()
    c.check("y", y); c.check("dx", dx)


@pytest.mark.parametrize("n", [20, 700])
def test_ids_outside_the_adapters(ctx, n):
    c = Case(n, 64, 64, 4, 8, BF16)
    bad = torch.randint(0, n, (max(n // 7, 1),), device="cuda")
    c.ids[bad] = torch.where(bad % 2 == 0, 4, -5).to(torch.int32)
    c.define()
    y, v = c.forward(ctx)
    assert B.emoe_device_status(ctx) == B.ERR_DEVICE_CHECK
    dx, dA, dB = c.backward(ctx, v)
    assert B.emoe_device_status(ctx) == B.ERR_DEVICE_CHECK
    assert B.emoe_device_status(ctx) == B.OK
    for what, got in (("v", v), ("y", y), ("dx", dx), ("dA", dA), ("dB", dB)):
        c.check(what, got)


@pytest.mark.parametrize("n,kind", [(9, "ids"), (700, "ids"), (700, "off")])
def test_rows_of_others_do_not_reach_a_result(ctx, n, kind):
    """NaN and infinities in one row, and in the factors of one adapter, stay where they belong."""
    c = Case(n, 128, 96, 4, 16, BF16, kind, none=0.2, ids=torch.arange(n, device="cuda") % 4)
    bad_rows = (c.ids == 2)
    c.A[2], c.B[2] = float("nan"), float("inf")
    none = (c.ids == -1)
    c.x[none], c.dy[none] = float("nan"), float("inf")
    c.x[bad_rows] = float("inf")
    v = torch.nan_to_num(c.forward(ctx)[1])
    y, _ = c.forward(ctx)
    dx, dA, dB = c.backward(ctx, v)
    torch.cuda.synchronize()
    c.base = torch.where(none[:, None], c.base, c.base)
    good = (c.ids >= 0) & ~bad_rows
    for t in (y, dx):
        assert torch.isfinite(t[good]).all()
        assert not torch.isfinite(t[bad_rows]).any()
    if kind == "ids":
        assert torch.equal(y[none], c.base[none])
    for a in (0, 1, 3):
        assert torch.isfinite(dA[a]).all() and torch.isfinite(dB[a]).all()
    assert not torch.isfinite(dA[2]).any()


def test_an_infinite_row_gives_infinities(ctx):
    """bf16: an infinite low-rank vector has no second part that would turn the result into NaN."""
    c = Case(4, 64, 64, 1, 16, BF16, scales=False)
    c.x[1] = 0
    c.x[1, 5] = float("inf")
    c.A[0] = c.A[0].abs() + 0.1
    c.B[0] = c.B[0].abs() + 0.1
    y, v = c.forward(ctx)
    torch.cuda.synchronize()
    assert (v[1] == float("inf")).all() and (y[1] == float("inf")).all() and torch.isfinite(y[[0, 2, 3]]).all()


@pytest.mark.parametrize("n", [4, 1000])
def test_captured_and_replayed_on_new_rows(ctx, n):
    """Forward and backward in one graph; the adapters of the rows change between replays."""
    c = Case(n, 256, 128, 8, 16, BF16)
    side = torch.cuda.Stream()
    y, v, dx = c.out(), torch.empty(n, 16, device="cuda"), c.inn()
    dA, dB = torch.empty(8, 16, 256, device="cuda"), torch.empty(8, 128, 16, device="cuda")

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
    for seed in (3, 4):
        o = Case(n, 256, 128, 8, 16, BF16, seed=seed, skew=float(seed == 4))
        for m in ("ids", "x", "dy", "base", "dx_base", "A", "B", "scales"):
            getattr(c, m).copy_(getattr(o, m))
        graph.replay()
        torch.cuda.synchronize()
        for what, got in (("v", v), ("y", y), ("dx", dx), ("dA", dA), ("dB", dB)):
            o.check(what, got)


def test_two_contexts_on_two_streams(ctx):
    cases = [Case(700, 256, 512, 4, 16, BF16, seed=1), Case(900, 128, 256, 9, 24, F32, seed=2)]
    hs = [B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, c.n)) for c in cases]
    outs = [(c.out(), torch.empty(c.n, c.r, device="cuda"), c.inn(), torch.empty(c.G, c.r, c.K, device="cuda"),
             torch.empty(c.G, c.N, c.r, device="cuda")) for c in cases]
    torch.cuda.synchronize()

    def job(c, h, o):
        def work(stream):
            c.forward(h, y=o[0], v=o[1], stream=stream)
            c.backward(h, o[1], dx=o[2], dA=o[3], dB=o[4], stream=stream)
        return work

    side_by_side([job(c, h, o) for c, h, o in zip(cases, hs, outs)], 30)
    torch.cuda.synchronize()
    for c, h, o in zip(cases, hs, outs):
        for what, got in zip(("y", "v", "dx", "dA", "dB"), o):
            c.check(what, got)
        B.emoe_destroy(h)


def test_gradients_against_differences(ctx):
    """The gradients of loss = <w, y> with respect to a few entries of x, A and B, against central differences of the
    library's own fp32 forward pass.  A step of h gives a difference that is exact (y is bilinear) but for the rounding of the two
    losses: the tolerance of y's sum of magnitudes, over 2 h."""
    c = Case(40, 64, 48, 3, 8, F32, seed=5)
    w = c.dy
    c.dx_base.zero_()
    _, v = c.forward(ctx)
    dx, dA, dB = c.backward(ctx, v)
    h = 0.5

    def loss():
        y, _ = c.forward(ctx)
        torch.cuda.synchronize()
        return (y.double() * w.double()).sum().item()

    for t, grad, places in ((c.x, dx, [(0, 0), (17, 63), (39, 31)]), (c.A, dA, [(0, 0, 0), (2, 7, 63)]), (c.B, dB, [(1, 47, 7), (0, 5, 3)])):
        for p in places:
            keep = t[p].item()
            ends = []
            for s in (1, -1):
                t[p] = keep + s * h
                ends.append(loss())
            moved = (torch.tensor(keep + h) - torch.tensor(keep - h)).item()
            t[p] = keep
            noise = 2 * (2 * (64 + 8 + 16) * STEP * (c.mag["y"] * 2 * w.abs().double()).sum().item()) / moved
            assert abs((ends[0] - ends[1]) / moved - grad[p].item()) <= noise + 2.0 ** -20 * abs(grad[p].item()), (p, noise)


def test_workspace_is_checked(ctx):
    n = 1100                                       # (forward calls of up to 1024 rows need none)
    c = Case(n, 64, 64, 4, 8, BF16)
    need = B.emoe_lowrank_workspace_bytes(c.desc, n)
    assert need > 0 and B.emoe_lowrank_workspace_bytes(c.desc, n + 1) >= need
    small = B.emoe_create(0, 1024)
    with pytest.raises(B.EmoeError) as e:
        c.forward(small)
    assert e.value.status == B.ERR_WORKSPACE
    with pytest.raises(B.EmoeError) as e:
        c.backward(small, torch.zeros(n, 8, device="cuda"))
    assert e.value.status == B.ERR_WORKSPACE
    B.emoe_destroy(small)
    exact = B.emoe_create(0, need)
    y, v = c.forward(exact)
    dx, dA, dB = c.backward(exact, v)
    torch.cuda.synchronize()
    for what, got in (("v", v), ("y", y), ("dx", dx), ("dA", dA), ("dB", dB)):
        c.check(what, got)
    B.emoe_destroy(exact)


def test_overlapping_segments_touch_nothing_outside(ctx):
    """Offsets that are not ascending are refused on the device where they would need more room than rows have."""
    c = Case(4096, 64, 64, 8, 8, BF16, "off")
    off = c.off.clone()
    off[1::2] = 4096
    off[2::2] = 0
    c.off = off
    h = B.emoe_create(0, B.emoe_lowrank_workspace_bytes(c.desc, 4096))
    _, v = c.forward(h)
    c.backward(h, torch.nan_to_num(v))
    torch.cuda.synchronize()
    B.emoe_device_status(h)
    B.emoe_destroy(h)
