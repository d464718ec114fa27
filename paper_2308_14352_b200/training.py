"""Device-memory plumbing around the calls for programs that train a sparse layer, or adapters beside one: rows in expert
order and back, the gates' gradient, low-rank adapters.  As in ``layer``, PyTorch only holds the memory; every step of the
computation is a call into libemoe.  Tensors are checked here (type, shape, device), since the library sees addresses only.
Calls go to the stream that torch works on at the time, whose memory their results are; a caller that names another stream orders the two.

One step of a layer with an adapter per expert, its experts frozen.  expert_outputs and through_experts are the experts' own products, forward and
back, in expert order: the program's, from experts that it holds unpacked (for packed ones there is no gradient call, and emoe_moe_forward gives the
gate-weighted sum alone):

    rows = er.dispatch(x, ids)                                       # expert order; er.off: first row of each expert
    out = ad.forward(rows, base=expert_outputs, off=er.off, keep=True)
    y = er.combine(out, gates)
    d_out, d_gates = er.combine_backward(dy, gates, out)
    d_rows, dA, dB = ad.backward(d_out, base=through_experts, off=er.off)
    dx, _ = er.dispatch_backward(d_rows)
    d_logits = gate_backward(ctx, logits, ids, d_gates, renorm)
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as B

_CODE = {torch.float32: B.DTYPE_F32, torch.bfloat16: B.DTYPE_BF16}


def _check(t: torch.Tensor, name: str, shape, dtype, device) -> torch.Tensor:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} "
                         f"on {t.device}" + ("" if t.is_contiguous() else ", not contiguous"))
    return t


def _gpu(ctx: int, device: torch.device, name: str) -> torch.device:
    if device.type != "cuda":
        raise ValueError(f"{name}: expected a tensor on a GPU, got one on {device}")
    if B.context_device(ctx) not in (None, device.index):
        raise ValueError(f"{name}: on {device}, but the context works on device {B.context_device(ctx)}")
    return device


def _stream(stream: Optional[int], device) -> int:
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class ExpertRows:
    """The order of one batch's (token, pick) pairs by expert, and the calls that use it.  ``dispatch`` sets the order that the
    other calls refer to: counts, off, perm and slots of the last batch."""

    def __init__(self, ctx: int, d: int, n_experts: int, top_k: int, token_dtype=torch.bfloat16, row_dtype=None, device: int = 0):
        self.ctx, self.d, self.n_experts, self.top_k = ctx, d, n_experts, top_k
        self.token_dtype, self.row_dtype = token_dtype, row_dtype or token_dtype
        if self.token_dtype not in _CODE or self.row_dtype not in _CODE:
            raise ValueError("tokens and rows are float32 or bfloat16")
        self.device = _gpu(ctx, torch.device("cuda", device), "rows")
        self.desc = B.emoe_dispatch_desc(d, n_experts, top_k, _CODE[self.token_dtype], _CODE[self.row_dtype], 0, 0, 0)
        self.tokens = 0  # of the last batch dispatched

    def _empty(self, *shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _tokens(self, t, name):
        if not self.tokens:
            raise ValueError("no batch has been dispatched")
        return _check(t, name, (self.tokens, self.d), self.token_dtype, self.device)

    def _rows(self, t, name):
        if not self.tokens:
            raise ValueError("no batch has been dispatched")
        return _check(t, name, (self.tokens * self.top_k, self.d), self.row_dtype, self.device)

    def _weights(self, t, name):
        return None if t is None else _check(t, name, (self.tokens, self.top_k), torch.float32, self.device)

    def dispatch(self, x: torch.Tensor, ids: torch.Tensor, weights: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> torch.Tensor:
        """Rows [tokens * top_k][d] in expert order, times the pairs' weights where given.  Rows of pairs without an expert (an id
        outside [0, n_experts): ``emoe_device_status`` tells) are not written."""
        tokens = x.shape[0]
        pairs = tokens * self.top_k
        _check(x, "x", (tokens, self.d), self.token_dtype, self.device)
        _check(ids, "ids", (tokens, self.top_k), torch.int32, self.device)
        if weights is not None:
            _check(weights, "weights", (tokens, self.top_k), torch.float32, self.device)
        counts, off = self._empty(self.n_experts, dtype=torch.int32), self._empty(self.n_experts + 1, dtype=torch.int32)
        perm, slots = self._empty(pairs, dtype=torch.int32), self._empty(pairs, dtype=torch.int32)
        rows = self._empty(pairs, self.d, dtype=self.row_dtype)
        B.emoe_dispatch(self.ctx, self.desc, x.data_ptr(), tokens, ids.data_ptr(), _ptr(weights), counts.data_ptr(), off.data_ptr(), perm.data_ptr(),
                        slots.data_ptr(), rows.data_ptr(), _stream(stream, self.device))
        self.tokens, self.counts, self.off, self.perm, self.slots = tokens, counts, off, perm, slots
        return rows

    def dispatch_backward(self, drows: torch.Tensor, weights: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None,
                          stream: Optional[int] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """(dx, gradient of the weights: only where x, the input of ``dispatch``, is given)."""
        self._rows(drows, "drows")
        dx = self._empty(self.tokens, self.d, dtype=self.token_dtype)
        dw = None if x is None else self._empty(self.tokens, self.top_k, dtype=torch.float32)
        B.emoe_dispatch_backward(self.ctx, self.desc, drows.data_ptr(), self.tokens, self.slots.data_ptr(),
                                 _ptr(self._weights(weights, "weights")), None if x is None else self._tokens(x, "x").data_ptr(), dx.data_ptr(),
                                 _ptr(dw), _stream(stream, self.device))
        return dx, dw

    def combine(self, rows: torch.Tensor, gates: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> torch.Tensor:
        self._rows(rows, "rows")
        y = self._empty(self.tokens, self.d, dtype=self.token_dtype)
        B.emoe_combine(self.ctx, self.desc, rows.data_ptr(), self.tokens, self.slots.data_ptr(),
                       _ptr(self._weights(gates, "gates")), y.data_ptr(), _stream(stream, self.device))
        return y

    def combine_backward(self, dy: torch.Tensor, gates: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                         stream: Optional[int] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """(drows, gradient of the gates: only where rows, the input of ``combine``, are given)."""
        self._tokens(dy, "dy")
        drows = self._empty(self.tokens * self.top_k, self.d, dtype=self.row_dtype)
        dg = None if rows is None else self._empty(self.tokens, self.top_k, dtype=torch.float32)
        B.emoe_combine_backward(self.ctx, self.desc, dy.data_ptr(), self.tokens, self.slots.data_ptr(),
                                _ptr(self._weights(gates, "gates")), None if rows is None else self._rows(rows, "rows").data_ptr(),
                                drows.data_ptr(), _ptr(dg), _stream(stream, self.device))
        return drows, dg


def gate_backward(ctx: int, logits: torch.Tensor, ids: torch.Tensor, dgates: torch.Tensor, renorm: bool, stream: Optional[int] = None) -> torch.Tensor:
    """Gradient of the router's logits from the gradient of its Top-K gates."""
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits are [tokens][experts], ids [tokens][picks]")
    T, E = logits.shape
    _gpu(ctx, logits.device, "logits")
    _check(logits, "logits", (T, E), torch.float32, logits.device)
    _check(ids, "ids", (T, ids.shape[1]), torch.int32, logits.device)
    _check(dgates, "dgates", ids.shape, torch.float32, logits.device)
    out = torch.empty_like(logits)
    B.emoe_gate_backward(ctx, logits.data_ptr(), T, E, ids.data_ptr(), dgates.data_ptr(), ids.shape[1],
                         B.GATE_SOFTMAX_RENORM if renorm else B.GATE_SOFTMAX, out.data_ptr(), _stream(stream, logits.device))
    return out


class LowRankAdapters:
    """Adapters A [n][rank][in], B [n][out][rank] (float32 or bfloat16) with a scale each, beside a shared projection."""

    def __init__(self, ctx: int, A: torch.Tensor, Bm: torch.Tensor, scales: Optional[torch.Tensor] = None):
        if A.dim() != 3 or Bm.dim() != 3 or A.dtype not in _CODE:
            raise ValueError("A is [adapters][rank][in], B [adapters][out][rank], float32 or bfloat16")
        self.ctx, self.device, self.dtype = ctx, _gpu(ctx, A.device, "A"), A.dtype
        self.n_adapters, self.rank, self.in_dim = A.shape
        self.out_dim = Bm.shape[1]
        self.A = _check(A, "A", A.shape, A.dtype, self.device)
        self.B = _check(Bm, "B", (self.n_adapters, self.out_dim, self.rank), A.dtype, self.device)
        self.scales = None if scales is None else _check(scales, "scales", (self.n_adapters,), torch.float32, self.device)
        self.desc = B.emoe_lowrank_desc(self.n_adapters, self.rank, self.in_dim, self.out_dim, _CODE[self.dtype], 0, 0, 0)
        self.x = self.v = None

    def workspace_bytes(self, rows: int) -> int:
        return B.emoe_lowrank_workspace_bytes(self.desc, rows)

    def _which(self, n, ids, off):
        if (ids is None) == (off is None):
            raise ValueError("either ids (an adapter per row) or off (first row of each adapter)")
        if ids is not None:
            return _check(ids, "ids", (n,), torch.int32, self.device).data_ptr(), None
        return None, _check(off, "off", (self.n_adapters + 1,), torch.int32, self.device).data_ptr()

    def forward(self, x: torch.Tensor, base: Optional[torch.Tensor] = None, ids: Optional[torch.Tensor] = None, off: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, keep: bool = False, stream: Optional[int] = None) -> torch.Tensor:
        """base + scale * B A x; `out` may be `base`.  With off, rows of no adapter are not written.  keep: x and the low-rank vectors stay here for ``backward``."""
        n = x.shape[0]
        _check(x, "x", (n, self.in_dim), self.dtype, self.device)
        which = self._which(n, ids, off)
        if base is not None:
            _check(base, "base", (n, self.out_dim), self.dtype, self.device)
        y = torch.empty(n, self.out_dim, dtype=self.dtype, device=self.device) if out is None else _check(out, "out", (n, self.out_dim), self.dtype,
                                                                                                          self.device)
        v = torch.empty(n, self.rank, dtype=torch.float32, device=self.device) if keep else None
        B.emoe_lowrank_forward(self.ctx, self.desc, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scales), x.data_ptr(), n, *which, _ptr(base),
                               y.data_ptr(), _ptr(v), _stream(stream, self.device))
        if keep:
            self.x, self.v = x, v
        return y

    def backward(self, dy: torch.Tensor, base: Optional[torch.Tensor] = None, ids: Optional[torch.Tensor] = None, off: Optional[torch.Tensor] = None,
                 stream: Optional[int] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(dx, dA, dB) of the last ``forward`` that kept its input; with off, rows of no adapter in dx are not written.
        base: the gradient of x that came through the shared projection."""
        if self.x is None:
            raise ValueError("backward needs a forward pass with keep=True")
        n = self.x.shape[0]
        _check(dy, "dy", (n, self.out_dim), self.dtype, self.device)
        which = self._which(n, ids, off)
        if base is not None:
            _check(base, "base", (n, self.in_dim), self.dtype, self.device)
        dx = torch.empty(n, self.in_dim, dtype=self.dtype, device=self.device)
        dA, dB = torch.empty_like(self.A, dtype=torch.float32), torch.empty_like(self.B, dtype=torch.float32)
        B.emoe_lowrank_backward(self.ctx, self.desc, self.A.data_ptr(), self.B.data_ptr(), _ptr(self.scales), self.x.data_ptr(), dy.data_ptr(), n, *which,
                                self.v.data_ptr(), _ptr(base), dx.data_ptr(), dA.data_ptr(), dB.data_ptr(), _stream(stream, self.device))
        return dx, dA, dB
