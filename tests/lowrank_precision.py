"""How far the low-rank calls' results may be from the formulas as a whole: one bound per result, tight enough that a value cut to fewer
bf16 parts than it has to be breaks it.

A result is a sum of products p of independent values of mean zero, and q = sqrt(sum p^2).  Over many results the norm of a partial sum of a
share f of the products is sqrt(f) |q|, so that errors relative to partial sums add up to a multiple of |q| that does not grow with the magnitudes'
sum.  In units of u = 2^-23, which is what the last place of an fp32 value is of it at most:
  tensor cores that add m instructions of sixteen products in one accumulator: each cuts the accumulator by less than u, in all less than
    sum_k sqrt(k / m) < 2 m / 3 + 1; and cuts sixteen products of either sign, together 4 u / sqrt(3) of the accumulator each time, independent:
    2.3 sqrt(m) x sqrt(1 / 2) < 4 sqrt(m).
  m sums of sixteen products that are added with rounding: half of u each at most: m / 3; the cuts within an instruction: 2.3 u of its sum, together
    2.3 u of q; products of parts that are left out: at most 2^-21 = 4 u of a product (both second parts below 2^-7, third ones below 2^-15).
  What else is rounded (shares of CTAs and runs, scales, a base that is added): less than 4 u.
So `cut(m)` = 2 m / 3 + 4 sqrt(m) + 8 and `rounded(m)` = m / 3 + 12.  A vector of which two truncated parts are left has lost 2^-16 of 1 .. 2 on
average, some 90 u of itself, with one part 2^-8, 23000 u."""
import math

import torch

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -23


def cut(m):
    return 2 * m / 3 + 4 * math.sqrt(m) + 8


def rounded(m):
    return m / 3 + 12


def parts_of(t, parts):
    """Values cut to their first bf16 parts, as the kernels cut fp32 values (truncated, so that three parts are the value)."""
    t = t.float()
    whole = torch.zeros_like(t)
    for _ in range(parts):
        part = ((t - whole).view(torch.int32) & -65536).view(F32)
        whole = whole + part
    return whole


class Inputs:
    """One call's tensors on `device` and its results in 64 bits; stream: (forward, backward) takes the kernels for many bf16 rows."""

    def __init__(self, n, K, N, G, r, dtype, stream=(False, False), device="cpu"):
        g = torch.Generator()
        g.manual_seed(17 * n + K + r)
        randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.n, self.K, self.N, self.G, self.r, self.dtype, self.stream = n, K, N, G, r, dtype, stream
        self.ids = torch.randint(0, G, (n,), generator=g, dtype=torch.int32).to(device)
        self.A, self.B = ((randn(*s) * f).to(dtype).to(device) for s, f in (((G, r, K), K ** -0.5), ((G, N, r), r ** -0.5)))
        self.scales = (torch.rand(G, generator=g) + 0.5).to(device)
        self.x, self.dy, self.base, self.dx_base = (randn(n, d).to(dtype).to(device) for d in (K, N, N, K))
        self.rows = [(self.ids == a).nonzero()[:, 0] for a in range(G)]
        self.most = max(len(at) for at in self.rows)
        self.ref = self.results()

    def results(self, vectors=None, values=None, rows=None, first=None):
        """v, y, dv, dx, dA, dB; `vectors` and `values`: bf16 parts of the vectors that enter a second product and of the tensors (None: whole).  first: only
        that many channels of the results (each is independent of the others)."""
        value = (lambda t: t.double()) if values is None else (lambda t: parts_of(t, values).double())
        vector = (lambda t: t) if vectors is None else (lambda t: parts_of(t, vectors).double())
        c = slice(0, first)
        f64 = dict(dtype=torch.float64, device=self.x.device)
        K, N = len(range(self.K)[c]), len(range(self.N)[c])
        out = {"v": torch.zeros(self.n, self.r, **f64), "dv": torch.zeros(self.n, self.r, **f64), "y": self.base[:, c].double().clone(),
               "dx": self.dx_base[:, c].double().clone(), "dA": torch.zeros(self.G, self.r, K, **f64), "dB": torch.zeros(self.G, N, self.r, **f64)}
        for a, at in enumerate(self.rows):
            A, Bm, x, dy, s = value(self.A[a]), value(self.B[a]), value(self.x[at]), value(self.dy[at]), self.scales[a].double()
            v, dv = x @ A.t(), s * (dy @ Bm)
            out["v"][at], out["dv"][at] = v, dv
            out["y"][at] += vector(s * v) @ Bm[c].t()
            out["dx"][at] += vector(dv) @ A[:, c]
            out["dA"][a] = vector(dv).t() @ x[:, c]
            out["dB"][a] = dy[:, c].t() @ vector(s * v)
        return out

    def bounds(self, first=None):
        """The bound of |result - formula| (2-norms) by result, in fp32; y and dx of bf16 tensors: without the rounding of the result."""
        c = slice(0, first)
        stream_f, stream_b = self.stream
        f32, channels = self.dtype == F32, 512 if self.r <= 32 else 256

        def down(dim, stream):   # (a cluster's warps share the channels: eight at least)
            return rounded(dim / 128 + 1) if f32 else cut(min(dim, channels) / 16) if stream else cut(dim / 128 + 1)

        c_v, c_dv = down(self.K, stream_f), down(self.N, stream_b)
        groups = math.ceil(min(self.most, 1024) / 16)
        outer = cut(groups) if stream_b else rounded(groups)
        up = rounded(math.ceil(self.r / 16)) if f32 else 2.0 ** -16 / U + 12   # bf16: two parts, the second rounded: 2^-16 of 1 .. 2
        q = {"v": 0.0, "dv": 0.0, "y": self.base[:, c].double().square().sum().item(), "dx": self.dx_base[:, c].double().square().sum().item(),
             "dA": 0.0, "dB": 0.0, "dA of dv": 0.0, "y of v": 0.0, "dx of dv": 0.0}
        for a, at in enumerate(self.rows):
            A, Bm, x, dy = (t.double().square() for t in (self.A[a], self.B[a], self.x[at], self.dy[at]))
            s = self.scales[a].double().square()
            v, dv = self.ref["v"][at].square(), self.ref["dv"][at].square()
            qv, qdv = x @ A.t(), s * (dy @ Bm)
            for name, t in (("v", qv), ("dv", qdv), ("y", s * v @ Bm[c].t()), ("y of v", s * qv @ Bm[c].t()), ("dx", dv @ A[:, c]),
                            ("dx of dv", qdv @ A[:, c]), ("dA", dv.t() @ x[:, c]), ("dA of dv", qdv.t() @ x[:, c]), ("dB", s * dy[:, c].t() @ v)):
                q[name] += t.sum().item()
        q = {k: math.sqrt(t) for k, t in q.items()}
        return {"v": U * c_v * q["v"], "y": U * (up * q["y"] + c_v * q["y of v"]), "dx": U * (up * q["dx"] + c_dv * q["dx of dv"]),
                "dA": U * (outer * q["dA"] + c_dv * q["dA of dv"]), "dB": U * (outer + 2) * q["dB"]}

    def cancel(self):
        """Bases that leave of y and dx what their type cannot hold of the sums, so that its rounding hides nothing of the sums' own errors."""
        for base, what in ((self.base, "y"), (self.dx_base, "dx")):
            low = self.ref[what] - base.double()
            base.copy_(-low)
        self.ref = self.results()


# n, K, N, adapters, rank, type, many rows (forward, backward).  Few rows per adapter: a short chain of sums, beside which two parts show; few
# channels down (N): vectors dv that are nearly exact themselves
CASES = [
    (4001, 2056, 64, 40, 16, BF16, (False, True)),
    (6000, 64, 2056, 50, 12, BF16, (False, True)),
    (3000, 2048, 136, 24, 32, BF16, (False, True)),
    (4000, 1032, 64, 40, 20, BF16, (False, True)),
    (2000, 2048, 72, 20, 64, BF16, (False, True)),
    (2500, 1544, 264, 25, 40, BF16, (False, True)),
    (4001, 2056, 64, 40, 5, BF16, (False, True)),
    (3001, 2056, 64, 30, 33, BF16, (False, True)),
    (4000, 2056, 4104, 40, 16, BF16, (True, True)),
    (1300, 4096, 8200, 13, 64, BF16, (True, True)),
    (9000, 1032, 2048, 1, 32, BF16, (True, True)),      # one adapter: whole runs, joined
    (37, 1104, 776, 5, 12, BF16, (False, False)),
    (900, 384, 640, 8, 16, BF16, (False, False)),
    (1024, 264, 136, 7, 24, BF16, (False, False)),
    (2100, 136, 128, 20, 64, BF16, (False, False)),
    (2100, 136, 128, 1, 8, BF16, (False, False)),
    (24, 768, 1024, 16, 8, F32, (False, False)),
    (130, 256, 512, 1, 64, F32, (False, False)),
    (200, 136, 96, 2, 33, F32, (False, False)),
    (515, 1104, 776, 5, 12, F32, (False, False)),
    (1000, 512, 512, 4, 64, F32, (False, False)),
    (2100, 264, 136, 3, 24, F32, (False, False)),
]
