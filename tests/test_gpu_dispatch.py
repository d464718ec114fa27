"""GPU parity: rows in expert order and back (emoe_dispatch, emoe_combine), their gradients, and the gradient of the gates,
against the definitions in 64 bits.  Tolerances: a result is a product or a sum of n products in fp32, whatever the order at
most n + 1 roundings of 2^-24 of the sum of the magnitudes, and one rounding of half a step to its own type."""
import numpy as np
import pytest
import torch

from paper_2308_14352_b200 import binding as B
from tests.helpers import side_by_side

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CODE = {F32: B.DTYPE_F32, BF16: B.DTYPE_BF16}


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 0)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


def _close(got, ref, magnitude, terms):
    """|got - ref| within half a step of got's type and (terms + 1) fp32 roundings of the sum of the magnitudes."""
    got, tol = got.double(), (terms + 1) * 2.0 ** -24 * magnitude + torch.finfo(got.dtype).eps / 2 * ref.abs() * (1 + 2.0 ** -8)
    assert torch.isfinite(got).all()
    worst = ((got - ref).abs() - tol).max().item()
    assert worst <= 1e-30, worst


def _strided(rows, d, dtype, pad, fill=None, offset=0):
    """A [rows][d] view with `pad` values behind each row and `offset` in front of the first."""
    base = torch.full((rows * (d + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    v = base[offset:].view(rows, d + pad)[:, :d]
    if fill is not None:
        v.copy_(fill)
    return v


class Case:
    def __init__(self, T, d, E, k, tok, row, weighted=True, bad=0.0, pad=(0, 0), offset=(0, 0), skew=0.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 7 * T + d)
        self.T, self.d, self.E, self.k, self.tok, self.row, self.P = T, d, E, k, tok, row, T * k
        self.pad, self.offset = pad, offset
        self.randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        p = torch.arange(1, E + 1, device="cuda", dtype=torch.float32) ** -skew
        self.ids = torch.multinomial(p.expand(T, E), k, generator=g, replacement=k > E).to(torch.int32)
        if bad:
            hit = torch.rand(T, k, generator=g, device="cuda") < bad
            self.ids[hit] = torch.where(torch.rand(int(hit.sum()), generator=g, device="cuda") < 0.5, -1, E + 3).to(torch.int32)
        self.w = self.randn(T, k).contiguous() if weighted else None
        self.x, self.dy = self.tokens(self.randn(T, d)), self.tokens(self.randn(T, d))
        self.drows = self.rows(self.randn(self.P, d))
        self.desc = B.emoe_dispatch_desc(d, E, k, CODE[tok], CODE[row], 0, d + pad[0] if pad[0] else 0, d + pad[1] if pad[1] else 0)
        # the definition
        flat = self.ids.flatten().long()
        ok = (flat >= 0) & (flat < E)
        key = torch.where(ok, flat, E)
        order = torch.sort(key, stable=True).indices[: int(ok.sum())]
        self.perm = torch.full((self.P,), -1, dtype=torch.int32, device="cuda")
        self.perm[: len(order)] = order.int()
        self.slots = torch.full((self.P,), -1, dtype=torch.int32, device="cuda")
        self.slots[order] = torch.arange(len(order), dtype=torch.int32, device="cuda")
        self.counts = torch.bincount(flat[ok], minlength=E).int()
        self.off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), self.counts.long().cumsum(0)]).int()
        self.owned = len(order)
        self.token = order // k
        self.w64 = torch.ones(self.P, dtype=torch.float64, device="cuda") if self.w is None else self.w.double().flatten()
        self.order = order

    def tokens(self, fill=None):
        return _strided(self.T, self.d, self.tok, self.pad[0], fill, self.offset[0])

    def rows(self, fill=None):
        return _strided(self.P, self.d, self.row, self.pad[1], fill, self.offset[1])

    def ptr(self, t):
        return None if t is None else t.data_ptr()

    def dispatch(self, ctx, stream=0, rows=None):
        rows = self.rows() if rows is None else rows
        e = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")  # noqa: E731
        out = dict(rows=rows, counts=e(self.E), off=e(self.E + 1), perm=e(self.P), slots=e(self.P))
        B.emoe_dispatch(ctx, self.desc, self.x.data_ptr(), self.T, self.ids.data_ptr(), self.ptr(self.w), out["counts"].data_ptr(),
                        out["off"].data_ptr(), out["perm"].data_ptr(), out["slots"].data_ptr(), rows.data_ptr(), stream)
        return out

    def check_dispatch(self, out):
        for m in ("counts", "off", "perm", "slots"):
            assert torch.equal(out[m], getattr(self, m)), m
        ref = self.w64[self.order, None] * self.x.double()[self.token]
        _close(out["rows"][: self.owned], ref, ref.abs(), 0)
        if self.w is None and self.tok == self.row:
            assert torch.equal(out["rows"][: self.owned], self.x[self.token])
        assert torch.isnan(out["rows"][self.owned:]).all()      # rows that no pair owns: as they were

    def gathered(self, rows, w):
        """sum over the picks of w * row, and the sum of the magnitudes."""
        t = w[self.order, None] * rows.double()[: self.owned]
        zero = lambda: torch.zeros(self.T, self.d, dtype=torch.float64, device="cuda")  # noqa: E731
        return zero().index_add_(0, self.token, t), zero().index_add_(0, self.token, t.abs())

    def products(self, rows, tokens):
        t = rows.double()[: self.owned] * tokens.double()[self.token]
        z = torch.zeros(self.P, dtype=torch.float64, device="cuda")
        return z.clone().index_add_(0, self.order, t.sum(1)), z.clone().index_add_(0, self.order, t.abs().sum(1))

    def check_back(self, ctx, stream=0):
        """The three calls that take slots."""
        dx, y, out = self.tokens(), self.tokens(), self.rows()
        dw, dg = (torch.full((self.T, self.k), float("nan"), device="cuda") for _ in range(2))
        clean = self.drows.clone()
        self.drows[self.owned:] = float("nan")                  # rows that no pair owns are not read
        w = self.ptr(self.w)
        B.emoe_dispatch_backward(ctx, self.desc, self.drows.data_ptr(), self.T, self.slots.data_ptr(), w, self.x.data_ptr(), dx.data_ptr(),
                                 dw.data_ptr(), stream)
        B.emoe_combine(ctx, self.desc, self.drows.data_ptr(), self.T, self.slots.data_ptr(), w, y.data_ptr(), stream)
        B.emoe_combine_backward(ctx, self.desc, self.dy.data_ptr(), self.T, self.slots.data_ptr(), w, self.drows.data_ptr(), out.data_ptr(),
                                dg.data_ptr(), stream)
        torch.cuda.synchronize()
        ref, mag = self.gathered(clean, self.w64)
        _close(dx, ref, mag, self.k)
        assert torch.equal(dx, y)                               # the same sum
        _close(dw.flatten(), *self.products(clean, self.x), self.d)
        _close(dg.flatten(), *self.products(clean, self.dy), self.d)
        ref = self.w64[self.order, None] * self.dy.double()[self.token]
        _close(out[: self.owned], ref, ref.abs(), 0)
        assert torch.isnan(out[self.owned:]).all()
        self.drows.copy_(clean)
        return dx, dw, dg, out


# T, d, E, k, tokens, rows, more
CASES = [
    (1, 4096, 8, 2, BF16, BF16, {}),
    (1, 1, 1, 1, F32, F32, {}),
    (2, 7, 256, 8, BF16, BF16, {"weighted": False}),
    (3, 64, 4, 4, F32, BF16, {"bad": 0.4}),
    (33, 1100, 32, 2, F32, F32, {}),
    (61, 1101, 5, 3, BF16, BF16, {}),                                    # rows of an odd number of bytes of any word
    (130, 100, 12, 5, BF16, F32, {"bad": 0.1}),
    (257, 8200, 3, 1, BF16, BF16, {"weighted": False}),                  # more pieces than one round of a CTA's threads
    (64, 2048, 8, 2, BF16, BF16, {"pad": (8, 16)}),                      # strides, still whole 16-byte words
    (64, 2048, 8, 2, BF16, F32, {"pad": (3, 5)}),                        # strides that are not
    (40, 512, 8, 2, BF16, BF16, {"offset": (1, 0)}),                     # rows of one side off the 16-byte boundary
    (40, 512, 8, 2, F32, BF16, {"offset": (0, 1)}),
    (40, 512, 8, 2, BF16, F32, {"offset": (4, 0)}),                      # 8-byte aligned tokens beside 16-byte rows: wide
    (1024, 96, 64, 2, F32, F32, {"skew": 1.1}),                          # the last size with order and rows in one launch
    (1025, 96, 64, 2, F32, F32, {"skew": 1.1}),                          # the first behind it
    (683, 40, 256, 3, BF16, BF16, {"bad": 0.3}),                         # 2049 pairs: a cluster of eight
    (5000, 72, 7, 8, BF16, F32, {"skew": 2.0, "bad": 0.01}),
    (9001, 24, 200, 1, F32, F32, {}),
    (16385, 16, 256, 8, BF16, BF16, {"weighted": False, "skew": 1.1}),   # several steps per warp of the order
    (4100, 8, 1, 1, BF16, BF16, {}),                                     # one expert
]


@pytest.mark.parametrize("T,d,E,k,tok,row,more", CASES)
def test_rows_and_their_gradients(ctx, T, d, E, k, tok, row, more):
    c = Case(T, d, E, k, tok, row, **more)
    out = c.dispatch(ctx)
    torch.cuda.synchronize()
    c.check_dispatch(out)
    assert B.emoe_device_status(ctx) == (B.ERR_DEVICE_CHECK if more.get("bad") and c.owned < c.P else B.OK)
    c.check_back(ctx)
    assert B.emoe_device_status(ctx) == B.OK


@pytest.mark.parametrize("T", [4, 2000])
def test_a_batch_without_any_expert(ctx, T):
    c = Case(T, 32, 4, 2, BF16, BF16)
    c.ids.fill_(-1)
    out = c.dispatch(ctx)
    torch.cuda.synchronize()
    assert out["counts"].sum() == 0 and out["off"].abs().sum() == 0
    assert (out["perm"] == -1).all() and (out["slots"] == -1).all() and torch.isnan(out["rows"]).all()
    assert B.emoe_device_status(ctx) == B.ERR_DEVICE_CHECK
    y = c.tokens()
    dg = torch.full((T, 2), float("nan"), device="cuda")
    B.emoe_combine(ctx, c.desc, out["rows"].data_ptr(), T, out["slots"].data_ptr(), c.w.data_ptr(), y.data_ptr(), 0)
    B.emoe_combine_backward(ctx, c.desc, c.dy.data_ptr(), T, out["slots"].data_ptr(), c.w.data_ptr(), out["rows"].data_ptr(),
                            out["rows"].data_ptr(), dg.data_ptr(), 0)
    torch.cuda.synchronize()
    assert (y == 0).all() and (dg == 0).all() and torch.isnan(out["rows"]).all()


def test_weights_of_dropped_pairs_and_infinities(ctx):
    """A dropped pair's weight is not used, whatever it is; an infinite row reaches its own token only."""
    c = Case(50, 64, 4, 2, F32, F32, bad=0.3)
    c.w[(c.slots.view(50, 2) < 0)] = float("nan")
    rows = c.randn(c.P, 64)
    rows[0, 3] = float("inf")
    y = c.tokens()
    B.emoe_combine(ctx, c.desc, rows.data_ptr(), 50, c.slots.data_ptr(), c.w.data_ptr(), y.data_ptr(), 0)
    torch.cuda.synchronize()
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[c.token[0], 3] = True
    assert torch.equal(torch.isinf(y), hit) and not torch.isnan(y).any()
    B.emoe_device_status(ctx)


def test_slots_outside_the_rows_are_dropped(ctx):
    """Whatever stands in slot_of_pair, no address outside [0, T*top_k) is touched."""
    c = Case(20, 48, 4, 2, BF16, BF16)
    slots = c.slots.clone()
    slots[3], slots[8], slots[39] = 40, 2 ** 31 - 1, -(2 ** 31)
    y = c.tokens()
    B.emoe_combine(ctx, c.desc, c.drows.data_ptr(), 20, slots.data_ptr(), c.w.data_ptr(), y.data_ptr(), 0)
    torch.cuda.synchronize()
    w = c.w64.clone()
    w[[3, 8, 39]] = 0
    ref, mag = c.gathered(c.drows, w)
    _close(y, ref, mag, 2)


def test_rows_may_be_overwritten_by_their_gradient(ctx):
    c = Case(300, 520, 8, 2, BF16, BF16)
    _, _, dg, out = c.check_back(ctx)
    rows, dg2 = c.drows.clone(), torch.empty_like(dg)
    B.emoe_combine_backward(ctx, c.desc, c.dy.data_ptr(), 300, c.slots.data_ptr(), c.w.data_ptr(), rows.data_ptr(), rows.data_ptr(), dg2.data_ptr(), 0)
    torch.cuda.synchronize()
    assert torch.equal(rows, out) and torch.equal(dg, dg2)


@pytest.mark.parametrize("T", [8, 3000])
def test_dispatch_in_a_captured_graph_follows_new_ids(ctx, T):
    c = Case(T, 128, 16, 2, BF16, BF16, weighted=False)
    side = torch.cuda.Stream()
    rows = c.rows()
    with torch.cuda.stream(side):
        c.dispatch(ctx, side.cuda_stream, rows)  # first launches outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = c.dispatch(ctx, side.cuda_stream, rows)
    for seed in (1, 2):
        other = Case(T, 128, 16, 2, BF16, BF16, weighted=False, seed=seed)
        c.ids.copy_(other.ids)
        c.x.copy_(other.x)
        graph.replay()
        torch.cuda.synchronize()
        other.check_dispatch(out)


def test_calls_on_two_streams_at_once(ctx):
    cases = [Case(2500, 256, 16, 2, BF16, BF16, seed=1), Case(700, 256, 16, 2, F32, F32, seed=2)]
    contexts = [B.emoe_create(0, 0) for _ in cases]
    outs = [c.dispatch(ctx) for c in cases]
    side_by_side([lambda s, c=c, o=o, h=h: B.emoe_dispatch(h, c.desc, c.x.data_ptr(), c.T, c.ids.data_ptr(), c.w.data_ptr(),
                                                           o["counts"].data_ptr(), o["off"].data_ptr(), o["perm"].data_ptr(),
                                                           o["slots"].data_ptr(), o["rows"].data_ptr(), s)
                  for c, o, h in zip(cases, outs, contexts)], 50)
    torch.cuda.synchronize()
    for c, o, h in zip(cases, outs, contexts):
        c.check_dispatch(o)
        B.emoe_destroy(h)


def test_rows_beyond_two_gigabytes(ctx):
    """Offsets of more than 32 bits: few tokens on rows that lie far apart."""
    T, d, stride = 9, 64, 1 << 27
    desc = B.emoe_dispatch_desc(d, 4, 2, B.DTYPE_BF16, B.DTYPE_BF16, 0, 0, stride)
    c = Case(T, d, 4, 2, BF16, BF16)
    big = torch.empty((2 * T - 1) * stride + d, dtype=BF16, device="cuda")
    e = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    slots, y = e(2 * T), c.tokens()
    B.emoe_dispatch(ctx, desc, c.x.data_ptr(), T, c.ids.data_ptr(), None, e(4).data_ptr(), e(5).data_ptr(), e(2 * T).data_ptr(), slots.data_ptr(),
                    big.data_ptr(), 0)
    B.emoe_combine(ctx, desc, big.data_ptr(), T, slots.data_ptr(), None, y.data_ptr(), 0)
    torch.cuda.synchronize()
    for s in range(2 * T):
        assert torch.equal(big[s * stride:s * stride + d], c.x[c.token[s]])
    assert torch.equal(y, (2 * c.x.float()).to(BF16))


# ---- gradient of the gates -----------------------------------------------------------------------

def _gate_ref(z, ids, dg, renorm):
    z, dg, E = z.double(), dg.double(), z.shape[1]
    ok = (ids >= 0) & (ids < E)
    at, dg = torch.where(ok, ids, 0).long(), torch.where(ok, dg, 0.0)
    if renorm:
        picked = torch.where(ok, z.gather(1, at), float("-inf"))
        top = picked.amax(1, keepdim=True)
        g = torch.where(ok & (top > float("-inf")), torch.exp(picked - torch.where(top > float("-inf"), top, 0.0)), 0.0)
        g = g / g.sum(1, keepdim=True).clamp_min(1e-300)
        return torch.zeros_like(z).scatter_add_(1, at, torch.where(ok, g * (dg - (g * dg).sum(1, keepdim=True)), 0.0))
    top = z.amax(1, keepdim=True)
    p = torch.where(top > float("-inf"), torch.exp(z - torch.where(top > float("-inf"), top, 0.0)), 0.0)
    p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    D = torch.zeros_like(z).scatter_add_(1, at, dg)
    return p * (D - (p * D).sum(1, keepdim=True))


def _gate(ctx, z, ids, dg, renorm, stream=0):
    T, E = z.shape
    dz = torch.full((T, E), float("nan"), device="cuda")
    B.emoe_gate_backward(ctx, z.data_ptr(), T, E, ids.data_ptr(), dg.data_ptr(), ids.shape[1], B.GATE_SOFTMAX_RENORM if renorm else B.GATE_SOFTMAX,
                         dz.data_ptr(), stream)
    torch.cuda.synchronize()
    return dz


def _gate_tolerance(z, dg):
    """p carries the rounding of z - max (2^-24 of its size), expf's 2 ulp, the sum of up to E + 1 terms and the division; dz adds as
    much again of |D| and the mean of D.  All relative to p <= 1 and |D| <= sum |dg|."""
    E = z.shape[1]
    span = torch.where(torch.isfinite(z), z, 0.0).abs().max().item()
    return (2 * E + 8 * span + 32) * 2.0 ** -24 * dg.abs().sum(1).max().item()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 4, 2), (3, 8, 8), (64, 32, 1), (257, 30, 3), (33, 64, 2), (500, 100, 4), (77, 127, 5), (1000, 128, 8),
                                   (19, 200, 8), (2049, 256, 2), (5, 255, 1), (31, 6, 6)])
@pytest.mark.parametrize("renorm", [False, True])
def test_gate_gradient(ctx, T, E, k, renorm):
    g = torch.Generator(device="cuda")
    g.manual_seed(T + E)
    z = torch.randn(T, E, generator=g, device="cuda") * 2
    ids = torch.topk(z, k, dim=1).indices.to(torch.int32).contiguous()
    dg = torch.randn(T, k, generator=g, device="cuda")
    dz = _gate(ctx, z, ids, dg, renorm)
    assert (dz.double() - _gate_ref(z, ids, dg, renorm)).abs().max().item() <= _gate_tolerance(z, dg)
    # against differences of the gates themselves, in 64 bits
    if T * E <= 8192:
        def loss(z64):
            p = torch.softmax(z64.gather(1, ids.long()), 1) if renorm else torch.softmax(z64, 1).gather(1, ids.long())
            return (p * dg.double()).sum(1)
        h = 1e-5
        for e in range(min(E, 8)):
            step = torch.zeros(1, E, dtype=torch.float64, device="cuda")
            step[0, e] = h
            fd = (loss(z.double() + step) - loss(z.double() - step)) / (2 * h)
            assert (fd - dz[:, e].double()).abs().max().item() <= _gate_tolerance(z, dg) + 1e-8 * dg.abs().sum(1).max().item()


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [8, 33, 256])
def test_gate_gradient_of_masked_and_odd_rows(ctx, renorm, E):
    g = torch.Generator(device="cuda")
    g.manual_seed(E)
    z = torch.randn(12, E, generator=g, device="cuda")
    ids = torch.topk(z, 3, dim=1).indices.to(torch.int32).contiguous()
    dg = torch.randn(12, 3, generator=g, device="cuda")
    z[0] = float("-inf")                                          # nothing left
    z[1, :] = float("-inf"); z[1, 2] = 0.5; ids[1] = torch.tensor([2, 0, 1])   # one expert left
    z[2, 4:] = float("-inf"); ids[2] = torch.tensor([0, 3, 1])
    z[3, 1:] = torch.finfo(F32).min; ids[3] = torch.tensor([0, 1, 2])          # masked by the type's lowest value
    z[4] = torch.finfo(F32).min                                   # ... all of them: an even softmax
    ids[5] = torch.tensor([3, 3, 3])                              # the same pick three times
    ids[6] = torch.tensor([-1, 2, E])                             # picks outside
    ids[7] = torch.tensor([-1, -1, E + 9])                        # no pick at all
    dg[6, 0] = float("nan")                                       # ... whatever their gradient is
    z[8] += 80; z[9] -= 90
    ref = _gate_ref(z, ids, dg, renorm)
    dz = _gate(ctx, z, ids, dg, renorm)
    assert B.emoe_device_status(ctx) == B.ERR_DEVICE_CHECK
    assert torch.isfinite(dz).all()
    clean = torch.nan_to_num(dg)
    for t in range(12):
        zt = z[t:t + 1] if t not in (3, 4) else torch.zeros(1, E, device="cuda")  # (differences of the lowest value are exact: 0 or it)
        assert (dz[t].double() - ref[t]).abs().max().item() <= _gate_tolerance(zt, clean[t:t + 1])
    assert (dz[0] == 0).all() and (dz[7] == 0).all()
