"""One training step of a sparse layer through the library's calls, run together as a program runs them: router, rows in
expert order, an adapter per expert beside the expert's own product, gate-weighted sum, and all the way back to the input, the router
logits and the adapters.  The reference is the same layer written with torch operations in 64 bits and differentiated by
torch; and central differences of the library's own forward pass."""
import pytest
import torch

from paper_2308_14352_b200 import binding as B, training

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    torch.zeros(1, device="cuda")
    c = B.emoe_create(0, 256 << 20)
    yield c
    torch.cuda.synchronize()
    B.emoe_destroy(c)


class Step:
    """T tokens of d values, E experts (a dense matrix each, frozen), top_k picks, adapters of `rank`."""

    def __init__(self, ctx, T, d, E, k, rank, dtype, renorm, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.ctx, self.T, self.d, self.E, self.k, self.renorm, self.dtype = ctx, T, d, E, k, renorm, dtype
        self.x, self.dy = randn(T, d).to(dtype), randn(T, d).to(dtype)
        self.Wr = randn(d, E) * d ** -0.5
        self.W = (randn(E, d, d) * d ** -0.5).to(dtype)
        self.A, self.Bm = (randn(E, rank, d) * d ** -0.5).to(dtype), (randn(E, d, rank) * 0.2).to(dtype)
        self.scales = torch.rand(E, generator=g, device="cuda") + 0.5

    def experts(self, rows, off, transposed=False):
        """The frozen experts' products, expert by expert (a program has its own way of doing this)."""
        out = torch.empty_like(rows)
        bounds = off.tolist()
        for e in range(self.E):
            at = slice(bounds[e], bounds[e + 1])
            w = self.W[e] if transposed else self.W[e].t()
            out[at] = (rows[at].double() @ w.double()).to(rows.dtype)
        return out

    def forward(self, x):
        T, E, k = self.T, self.E, self.k
        self.ids = torch.empty(T, k, dtype=torch.int32, device="cuda")
        self.gates, self.logits = torch.empty(T, k, device="cuda"), torch.empty(T, E, device="cuda")
        B.emoe_router_topk(self.ctx, x.data_ptr(), B.DTYPE_BF16 if self.dtype == torch.bfloat16 else B.DTYPE_F32, T, self.d, self.Wr.data_ptr(), None, 0,
                           E, k, B.GATE_SOFTMAX_RENORM if self.renorm else B.GATE_SOFTMAX, self.ids.data_ptr(), self.gates.data_ptr(),
                           self.logits.data_ptr(), 0)
        self.er = training.ExpertRows(self.ctx, self.d, E, k, self.dtype)
        self.ad = training.LowRankAdapters(self.ctx, self.A, self.Bm, self.scales)
        rows = self.er.dispatch(x, self.ids)
        self.out = self.ad.forward(rows, base=self.experts(rows, self.er.off), off=self.er.off, keep=True)
        return self.er.combine(self.out, self.gates)

    def backward(self, dy):
        dout, dgates = self.er.combine_backward(dy, self.gates, self.out)
        drows, dA, dB = self.ad.backward(dout, base=self.experts(dout, self.er.off, True), off=self.er.off)
        dx, _ = self.er.dispatch_backward(drows)
        dlogits = training.gate_backward(self.ctx, self.logits, self.ids, dgates, self.renorm)
        return {"dx": dx, "dlogits": dlogits, "dA": dA, "dB": dB, "dgates": dgates}

    def reference(self):
        """64 bits; x enters the experts' path and the logits separately, so that dx is the experts' path alone (as the library's is)."""
        x = self.x.double().requires_grad_()
        logits = self.logits.double().requires_grad_()
        A, Bm = self.A.double().requires_grad_(), self.Bm.double().requires_grad_()
        at = self.ids.long()
        picked = logits.gather(1, at)
        gates = torch.softmax(picked, 1) if self.renorm else torch.softmax(logits, 1).gather(1, at)
        every = torch.einsum("td,eod->teo", x, self.W.double())
        v = torch.einsum("td,erd->ter", x, A)
        every = every + self.scales.double()[None, :, None] * torch.einsum("ter,eor->teo", v, Bm)
        y = (gates[:, :, None] * every.gather(1, at[:, :, None].expand(-1, -1, self.d))).sum(1)
        (y * self.dy.double()).sum().backward()
        return y.detach(), {"dx": x.grad, "dlogits": logits.grad, "dA": A.grad, "dB": Bm.grad}


@pytest.mark.parametrize("T,d,E,k,rank,dtype,renorm", [
    (1, 64, 4, 2, 8, torch.float32, True),
    (37, 136, 5, 2, 5, torch.float32, False),
    (200, 256, 8, 1, 16, torch.float32, False),
    (300, 128, 16, 4, 12, torch.float32, True),
    (1500, 264, 6, 2, 16, torch.float32, True),
])
def test_a_step_in_fp32(ctx, T, d, E, k, rank, dtype, renorm):
    """Everything is fp32 here: each stage is off by the roundings of its sums (at most 2 d + 2 T of them in a row, doubled for sums that the tensor
    cores cut), relative to the largest magnitudes that meet in a result, which are bounded by the result's norm times d."""
    s = Step(ctx, T, d, E, k, rank, dtype, renorm, seed=T)
    y = s.forward(s.x)
    got = s.backward(s.dy)
    torch.cuda.synchronize()
    assert B.emoe_device_status(ctx) == B.OK
    y_ref, ref = s.reference()
    for name, a, b in [("y", y, y_ref)] + [(n, got[n], ref[n]) for n in ref]:
        scale = b.abs().max().item() if name != "dlogits" else s.dy.double().norm(dim=1).max().item() * s.out.double().norm(dim=1).max().item()
        err = (a.double() - b).abs().max().item()
        assert err <= 4 * (d + T) * STEP * scale * 4, (name, err, scale)


@pytest.mark.parametrize("T,d,E,k,rank,renorm", [(64, 256, 8, 2, 16, True), (3000, 1024, 8, 2, 16, True), (2500, 1032, 6, 1, 64, False)])
def test_a_step_in_bf16(ctx, T, d, E, k, rank, renorm):
    """bf16 rows: four tensors of the way (the experts' products, the rows behind the adapters, the two gradients that go back) are rounded to
    bf16, half a step of 2^-8 relative each, at random signs: in the 2-norm no more than their sum."""
    s = Step(ctx, T, d, E, k, rank, torch.bfloat16, renorm, seed=T)
    y = s.forward(s.x)
    got = s.backward(s.dy)
    torch.cuda.synchronize()
    assert B.emoe_device_status(ctx) == B.OK
    y_ref, ref = s.reference()
    for name, a, b in [("y", y, y_ref)] + [(n, got[n], ref[n]) for n in ref]:
        if k == 1 and renorm and name == "dlogits":
            continue
        err = ((a.double() - b).norm() / b.norm()).item()
        assert err <= 4 * 2.0 ** -8, (name, err)


def test_a_step_against_differences(ctx):
    """d(loss)/d(logit), d(loss)/dA and d(loss)/dx of the chain against central differences of the library's forward pass in fp32 (loss = <dy, y>
    summed in 64 bits).  x moves the experts' path alone: its difference is taken with the picks and gates held."""
    s = Step(ctx, 24, 64, 4, 2, 8, torch.float32, True, seed=3)
    s.forward(s.x)
    got = s.backward(s.dy)
    ids, gates = s.ids.clone(), s.gates.clone()

    def loss(x, A, Bm):
        ad = training.LowRankAdapters(ctx, A, Bm, s.scales)
        er = training.ExpertRows(ctx, s.d, s.E, s.k, s.dtype)
        rows = er.dispatch(x, ids)
        y = er.combine(ad.forward(rows, base=s.experts(rows, er.off), off=er.off), gates)
        return (y.double() * s.dy.double()).sum().item()

    size = (s.dy.double().abs().sum(1) * s.out.double().abs().amax()).sum().item() * s.k   # magnitudes that meet in the loss
    h = 0.25
    for name, t, places in (("dx", s.x, [(0, 0), (11, 63), (23, 30)]), ("dA", s.A, [(0, 0, 0), (3, 7, 63)]), ("dB", s.Bm, [(1, 63, 7), (2, 5, 3)])):
        for p in places:
            keep, ends = t[p].item(), []
            for sign in (1, -1):
                t[p] = keep + sign * h
                ends.append(loss(s.x, s.A, s.Bm))
            moved = (torch.tensor(keep + h) - torch.tensor(keep - h)).item()
            t[p] = keep
            slope = (ends[0] - ends[1]) / moved
            assert abs(slope - got[name][p].item()) <= 64 * STEP * size / moved, (name, p)   # y is linear in each of them: no truncation


def test_wrong_tensors_are_refused(ctx):
    er = training.ExpertRows(ctx, 64, 4, 2)
    x = torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    for bad in (lambda: er.dispatch(x.float(), ids), lambda: er.dispatch(x, ids.long()), lambda: er.dispatch(x[:, :32], ids),
                lambda: er.dispatch(x, ids[:2]), lambda: er.dispatch(x.cpu(), ids), lambda: er.dispatch(x.t().contiguous().t(), ids),
                lambda: er.combine(torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        training.ExpertRows(ctx, 64, 4, 2, torch.float16)
    A, Bm = torch.zeros(2, 8, 64, device="cuda"), torch.zeros(2, 16, 8, device="cuda")
    ad = training.LowRankAdapters(ctx, A, Bm)
    x = torch.zeros(3, 64, device="cuda")
    who = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (lambda: ad.forward(x), lambda: ad.forward(x, ids=who, off=who), lambda: ad.forward(x, ids=who[:2]), lambda: ad.forward(x, off=who[:2]),
                lambda: ad.forward(x, base=torch.zeros(3, 8, device="cuda"), ids=who), lambda: ad.backward(torch.zeros(3, 16, device="cuda"), ids=who),
                lambda: training.LowRankAdapters(ctx, A, Bm.transpose(1, 2))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.EmoeError) as e:
        er2 = training.ExpertRows(ctx, 64, 4, 2)
        er2.dispatch(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    assert e.value.status == B.ERR_INVALID_ARG
