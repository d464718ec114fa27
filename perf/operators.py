"""Measured operators beside the packed forward: what a program that trains or adapts a sparse layer, or serves many
adapters of one model, has this library do.

dispatch       tokens sorted by expert: the order and the rows in it, optionally times a weight per (token, expert) pair
dispatch_grad  its gradient: the copies of a token added up; with weights, the gradient of each weight too
combine        the rows back in token order, added with the pairs' gates
combine_grad   its gradient: rows and gates
gate_grad      gradient of the router's logits from the gradient of the Top-K gates
lowrank        y = base + s B (A x) with the adapter of each row's request (or expert); base is the shared projection's output
lowrank_grad   its gradient: dx, dA and dB

Shapes are those of the repository's workloads (inputs.WORKLOADS) and the ranges around them.  Activations and gradients
~ N(0, 1), gates are Top-K softmax values, A ~ N(0, 1 / in), B ~ N(0, 0.02^2).
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}


def _rows(name, work, tokens, d, experts, top_k, dtype="bf16", out="", weighted=False, skew=0.0):
    """dispatch and combine; `dtype`: type of the rows, `out`: of the tokens (where it differs)."""
    case = {"work": work, "tokens": tokens, "d": d, "experts": experts, "top_k": top_k, "dtype": dtype, "tokens_dtype": out or dtype,
            "weighted": weighted, "skew": skew}
    return dict(case, name=name) if name else case


def _gate(name, tokens, experts, top_k, renorm):
    case = {"work": "gate_grad", "tokens": tokens, "experts": experts, "top_k": top_k, "renorm": renorm}
    return dict(case, name=name) if name else case


def _lowrank(name, work, rows, k, n, adapters, rank, dtype="bf16", sorted_rows=False, save=False, skew=0.0):
    case = {"work": work, "rows": rows, "in": k, "out": n, "adapters": adapters, "rank": rank, "dtype": dtype, "sorted": sorted_rows,
            "save": save, "skew": skew}
    return dict(case, name=name) if name else case


def listed():
    return [
        # four requests decoding on a Mixtral-like layer whose experts the program multiplies itself: latency and launches
        _rows("dispatch_decode_t4", "dispatch", 4, 4096, 8, 2),
        # a training batch on that layer
        _rows("dispatch_mixtral_t8192", "dispatch", 8192, 4096, 8, 2),
        # fp32 training of a small model, rows of no round size, pair weights applied on the way in
        _rows("dispatch_grad_f32_t2039", "dispatch_grad", 2039, 1100, 32, 2, "f32", weighted=True),
        # prefill over 128 experts with Zipf-like loads, bf16 expert outputs into the fp32 residual
        _rows("combine_zipf_t2048", "combine", 2048, 1024, 128, 1, "bf16", "f32", skew=1.1),
        # fine-grained experts, eight per token: the widest gather
        _rows("combine_k8_t16384", "combine", 16384, 2048, 128, 8),
        # the backward pass of the Mixtral-like training batch
        _rows("combine_grad_mixtral_t8192", "combine_grad", 8192, 4096, 8, 2),
        # router gradient of a served-size batch on a Switch-base layer, and of a long odd one with eight picks
        _gate("gate_grad_switch_t64", 64, 32, 1, False),
        _gate("gate_grad_k8_t16411", 16411, 128, 8, False),
        # one decoding step of 24 requests over 16 adapters beside an attention-sized projection
        _lowrank("lowrank_decode_n24", "lowrank", 24, 4096, 4096, 16, 16),
        # prompts of many adapters, an odd number of rows, beside a gated up-projection
        _lowrank("lowrank_prefill_n4099", "lowrank", 4099, 4096, 14336, 16, 32, skew=1.1),
        # fp32 adapters of ragged sizes, low-rank vectors kept for the backward pass
        _lowrank("lowrank_f32_n515", "lowrank", 515, 1104, 776, 5, 12, "f32", save=True),
        # one adapter per expert on rows that dispatch has sorted: the backward pass of a training batch
        _lowrank("lowrank_grad_experts_n8192", "lowrank_grad", 8192, 4096, 4096, 8, 16, sorted_rows=True, skew=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["dispatch", "dispatch", "dispatch_grad", "combine", "combine", "combine_grad", "gate_grad", "lowrank", "lowrank",
                       "lowrank", "lowrank_grad", "lowrank_grad"])
    if kind == "gate_grad":
        experts = rng.choice([4, 8, 30, 32, 64, 128, 200, 256])
        return _gate(None, _log_int(rng, 1, 32768), experts, rng.randint(1, min(8, experts)), rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("lowrank"):
        step = rng.choice([8, 32, 128])
        k, n = (step * _log_int(rng, max(256, step) // step, 8192 // step) for _ in range(2))
        adapters, rank = _log_int(rng, 1, 64), rng.choice([4, 8, 12, 16, 16, 32, 64])
        most = 100e6 / ((k + n) * _SIZE[dtype])
        rows = _log_int(rng, 1, min(16384, most)) if kind == "lowrank" else _log_int(rng, 64, max(65, min(8192, most)))
        return _lowrank(None, kind, rows, k, n, adapters, rank, dtype, rng.random() < (0.3 if kind == "lowrank" else 0.6),
                        kind == "lowrank" and rng.random() < 0.3, rng.choice([0.0, 0.5, 1.1]))
    experts = rng.choice([4, 8, 16, 32, 64, 128, 256])
    top_k = rng.choice([1, 1, 2, 2, 4, 8] if experts >= 8 else [1, 2])
    d = _log_int(rng, 16, 6144) if rng.random() < 0.3 else 128 * _log_int(rng, 3, 48)
    tokens = _log_int(rng, 1, min(32768, 200e6 / (d * (top_k + 1) * _SIZE[dtype])))
    out = rng.choice(["bf16", "f32"]) if kind.startswith("combine") else dtype
    return _rows(None, kind, tokens, d, experts, top_k, dtype, out, kind.startswith("dispatch") and rng.random() < 0.5, rng.choice([0.0, 0.0, 1.1]))


# ---- inputs ----------------------------------------------------------------------------------


def _ids(gen, tokens, experts, top_k, skew):
    """top_k different experts per token, expert e with weight (e + 1)^-skew, in no order."""
    bias = -skew * torch.log(torch.arange(1, experts + 1, device="cuda", dtype=torch.float32))
    noise = -torch.log(-torch.log(torch.rand(tokens, experts, generator=gen, device="cuda").clamp_(1e-9, 1 - 1e-7)))
    return torch.topk(noise + bias, top_k, dim=1).indices.to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    s = dict(case)
    if case["work"] == "gate_grad":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        s["logits"] = randn(T, E) * 1.5
        s["ids"] = torch.topk(s["logits"], k, dim=1).indices.to(torch.int32).contiguous()
        s["dgates"] = randn(T, k)
        s["dlogits"] = empty((T, E), torch.float32)
        return s
    dt = _TYPES[case["dtype"]]
    if case["work"].startswith("lowrank"):
        n, K, N, G, r = case["rows"], case["in"], case["out"], case["adapters"], case["rank"]
        ids = _ids(gen, n, G, 1, case["skew"])[:, 0].contiguous()
        if case["sorted"]:
            ids = torch.sort(ids).values.contiguous()
            s["off"] = torch.searchsorted(ids, torch.arange(G + 1, device="cuda", dtype=torch.int32)).to(torch.int32)
        else:
            s["ids"] = ids
        s["A"] = (randn(G, r, K) / math.sqrt(K)).to(dt)
        s["B"] = (randn(G, N, r) * 0.02).to(dt)
        s["scales"] = torch.rand(G, generator=gen, device="cuda") + 0.5
        s["x"] = randn(n, K).to(dt)
        if case["work"] == "lowrank":
            s["base"] = randn(n, N).to(dt)
            s["y"] = empty((n, N), dt)
            s["v"] = empty((n, r), torch.float32) if case["save"] else None
            return s
        # what the forward pass has kept, and the gradients that come from behind it
        every = (s["x"].float() @ s["A"].float().view(G * r, K).t()).view(n, G, r)
        s["v"] = every[torch.arange(n, device="cuda"), ids.long()].contiguous()
        s["dy"] = randn(n, N).to(dt)
        s["dx_base"] = randn(n, K).to(dt)
        s["dx"] = empty((n, K), dt)
        s["dA"] = empty((G, r, K), torch.float32)
        s["dB"] = empty((G, N, r), torch.float32)
        return s
    T, d, E, k = case["tokens"], case["d"], case["experts"], case["top_k"]
    P, tt = T * k, _TYPES[case["tokens_dtype"]]
    ids = _ids(gen, T, E, k, case["skew"])
    weights = torch.softmax(randn(T, k), dim=1).contiguous() if case["weighted"] or case["work"].startswith("combine") else None
    s["weights"] = weights
    if case["work"] == "dispatch":
        s.update(x=randn(T, d).to(tt), ids=ids, rows=empty((P, d), dt), counts=empty(E, torch.int32), off=empty(E + 1, torch.int32),
                 perm=empty(P, torch.int32), slots=empty(P, torch.int32))
        return s
    # the order of the forward pass
    order = torch.sort(ids.flatten(), stable=True).indices
    s["slots"] = empty(P, torch.int32)
    s["slots"][order] = torch.arange(P, dtype=torch.int32, device="cuda")
    if case["work"] == "combine":
        s.update(rows=randn(P, d).to(dt), y=empty((T, d), tt))
    elif case["work"] == "combine_grad":
        s.update(rows=randn(P, d).to(dt), dy=randn(T, d).to(tt), drows=empty((P, d), dt), dgates=empty((T, k), torch.float32))
    else:
        s.update(drows=randn(P, d).to(dt), x=randn(T, d).to(tt) if weights is not None else None, dx=empty((T, d), tt),
                 dweights=empty((T, k), torch.float32) if weights is not None else None)
    return s


# ---- plain forms -----------------------------------------------------------------------------


def _plain_rows(s):
    T, k = s["tokens"], s["top_k"]
    w = s["weights"]
    if s["work"] == "dispatch":
        flat = s["ids"].flatten()
        perm = torch.argsort(flat, stable=True)
        slots = torch.empty_like(perm)
        slots[perm] = torch.arange(T * k, device=flat.device)
        counts = (flat[:, None] == torch.arange(s["experts"], device=flat.device)).sum(0)
        off = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        rows = s["x"][perm // k]
        if w is not None:
            rows = (rows.float() * w.flatten()[perm][:, None]).to(s["rows"].dtype)
        return {"rows": rows, "counts": counts.int(), "off": off.int(), "perm": perm.int(), "slots": slots.int()}
    at = s["slots"].long()
    if s["work"] == "combine":
        return {"y": (s["rows"].float()[at].view(T, k, -1) * w[:, :, None]).sum(1).to(s["y"].dtype)}
    if s["work"] == "combine_grad":
        dy = s["dy"].float()
        drows = torch.empty_like(s["drows"])
        drows[at] = (dy[:, None, :] * w[:, :, None]).view(T * k, -1).to(drows.dtype)
        return {"drows": drows, "dgates": (s["rows"].float()[at].view(T, k, -1) * dy[:, None, :]).sum(-1)}
    back = s["drows"].float()[at].view(T, k, -1)
    if w is None:
        return {"dx": back.sum(1).to(s["dx"].dtype)}
    return {"dx": (back * w[:, :, None]).sum(1).to(s["dx"].dtype), "dweights": (back * s["x"].float()[:, None, :]).sum(-1)}


def _plain_gate(s):
    z, at, dg = s["logits"], s["ids"].long(), s["dgates"]
    if s["renorm"]:
        g = torch.exp(z.gather(1, at) - z.amax(1, keepdim=True))
        g = g / g.sum(1, keepdim=True)
        return {"dlogits": torch.zeros_like(z).scatter_add(1, at, g * (dg - (g * dg).sum(1, keepdim=True)))}
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    of_expert = torch.zeros_like(z).scatter_add(1, at, dg)
    return {"dlogits": p * (of_expert - (of_expert * p).sum(1, keepdim=True))}


def _plain_lowrank(s):
    """All adapters' products at once, those of other rows' adapters set to zero."""
    G, r, K, N = s["adapters"], s["rank"], s["in"], s["out"]
    each = torch.arange(G, device=s["x"].device)
    if s["sorted"]:
        row = torch.arange(s["rows"], device=s["x"].device)[:, None]
        mine = (row >= s["off"][:-1]) & (row < s["off"][1:])
    else:
        mine = s["ids"][:, None] == each
    mine = mine.float().repeat_interleave(r, dim=1)
    scales = s["scales"].repeat_interleave(r)
    A = s["A"].float().view(G * r, K)
    Bt = s["B"].float().transpose(1, 2).reshape(G * r, N)
    x = s["x"].float()
    if s["work"] == "lowrank":
        v = (x @ A.t()) * mine
        out = {"y": (s["base"].float() + (v * scales) @ Bt).to(s["y"].dtype)}
        if s["save"]:
            out["v"] = v.view(-1, G, r).sum(1)
        return out
    dy = s["dy"].float()
    v = s["v"].repeat(1, G) * mine * scales
    dv = (dy @ Bt.t()) * mine * scales
    return {"dx": (s["dx_base"].float() + dv @ A).to(s["dx"].dtype), "dA": (dv.t() @ x).view(G, r, K),
            "dB": (v.t() @ dy).view(G, r, N).transpose(1, 2).contiguous()}


# ---- the framework's calls -------------------------------------------------------------------

_handle = {}


def _library():
    """The program's one context, with room for the largest call of the ranges above."""
    if not _handle:
        from paper_2308_14352_b200 import binding as B

        most = B.emoe_lowrank_desc(64, 64, 14336, 14336, B.DTYPE_BF16, 0, 0, 0)
        _handle.update(B=B, ctx=B.emoe_create(torch.cuda.current_device(), B.emoe_lowrank_workspace_bytes(most, 16384)),
                       dtype={torch.float32: B.DTYPE_F32, torch.bfloat16: B.DTYPE_BF16})
    return _handle


def _ptr(t):
    return None if t is None else t.data_ptr()


def _own_rows(s):
    h = _library()
    B, ctx, stream = h["B"], h["ctx"], torch.cuda.current_stream().cuda_stream
    desc = B.emoe_dispatch_desc(s["d"], s["experts"], s["top_k"], h["dtype"][_TYPES[s["tokens_dtype"]]], h["dtype"][_TYPES[s["dtype"]]], 0, 0, 0)
    T, w = s["tokens"], _ptr(s["weights"])
    if s["work"] == "dispatch":
        B.emoe_dispatch(ctx, desc, s["x"].data_ptr(), T, s["ids"].data_ptr(), w, s["counts"].data_ptr(), s["off"].data_ptr(),
                        s["perm"].data_ptr(), s["slots"].data_ptr(), s["rows"].data_ptr(), stream)
        return {m: s[m] for m in ("rows", "counts", "off", "perm", "slots")}
    if s["work"] == "combine":
        B.emoe_combine(ctx, desc, s["rows"].data_ptr(), T, s["slots"].data_ptr(), w, s["y"].data_ptr(), stream)
        return {"y": s["y"]}
    if s["work"] == "combine_grad":
        B.emoe_combine_backward(ctx, desc, s["dy"].data_ptr(), T, s["slots"].data_ptr(), w, s["rows"].data_ptr(), s["drows"].data_ptr(),
                                s["dgates"].data_ptr(), stream)
        return {"drows": s["drows"], "dgates": s["dgates"]}
    B.emoe_dispatch_backward(ctx, desc, s["drows"].data_ptr(), T, s["slots"].data_ptr(), w, _ptr(s["x"]), s["dx"].data_ptr(),
                             _ptr(s["dweights"]), stream)
    return {"dx": s["dx"]} if w is None else {"dx": s["dx"], "dweights": s["dweights"]}


def _own_gate(s):
    h = _library()
    B = h["B"]
    B.emoe_gate_backward(h["ctx"], s["logits"].data_ptr(), s["tokens"], s["experts"], s["ids"].data_ptr(), s["dgates"].data_ptr(), s["top_k"],
                         B.GATE_SOFTMAX_RENORM if s["renorm"] else B.GATE_SOFTMAX, s["dlogits"].data_ptr(),
                         torch.cuda.current_stream().cuda_stream)
    return {"dlogits": s["dlogits"]}


def _own_lowrank(s):
    h = _library()
    B, ctx, stream = h["B"], h["ctx"], torch.cuda.current_stream().cuda_stream
    desc = B.emoe_lowrank_desc(s["adapters"], s["rank"], s["in"], s["out"], h["dtype"][_TYPES[s["dtype"]]], 0, 0, 0)
    ids, off = _ptr(s.get("ids")), _ptr(s.get("off"))
    if s["work"] == "lowrank":
        B.emoe_lowrank_forward(ctx, desc, s["A"].data_ptr(), s["B"].data_ptr(), s["scales"].data_ptr(), s["x"].data_ptr(), s["rows"], ids, off,
                               s["base"].data_ptr(), s["y"].data_ptr(), _ptr(s["v"]), stream)
        return {"y": s["y"], "v": s["v"]} if s["save"] else {"y": s["y"]}
    B.emoe_lowrank_backward(ctx, desc, s["A"].data_ptr(), s["B"].data_ptr(), s["scales"].data_ptr(), s["x"].data_ptr(), s["dy"].data_ptr(),
                            s["rows"], ids, off, s["v"].data_ptr(), s["dx_base"].data_ptr(), s["dx"].data_ptr(), s["dA"].data_ptr(),
                            s["dB"].data_ptr(), stream)
    return {m: s[m] for m in ("dx", "dA", "dB")}


def run(state):
    if state["work"] == "gate_grad":
        return _own_gate(state) if own else _plain_gate(state)
    if state["work"].startswith("lowrank"):
        return _own_lowrank(state) if own else _plain_lowrank(state)
    return _own_rows(state) if own else _plain_rows(state)


# ---- sizes and the definition in 64 bits -----------------------------------------------------


def work(case):
    if case["work"] == "gate_grad":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": 4.0 * T * (E + (k if case["renorm"] else E) + 2 * k), "flops": 0.0}
    z = _SIZE[case["dtype"]]
    if case["work"].startswith("lowrank"):
        n, K, N, G, r = case["rows"], case["in"], case["out"], case["adapters"], case["rank"]
        factors = min(n, G) * r * (K + N)
        flops = 2.0 * n * r * (K + N)
        if case["work"] == "lowrank":
            return {"bytes": float(z * (n * (K + 2 * N) + factors) + 4 * n * (r if case["save"] else 0)), "flops": flops}
        return {"bytes": float(z * (n * (3 * K + N) + factors) + 4 * (G * r * (K + N) + n * r)), "flops": 2 * flops}
    T, d, k, t = case["tokens"], case["d"], case["top_k"], _SIZE[case["tokens_dtype"]]
    P = T * k
    row, token = float(P * d * z), float(T * d * t)
    if case["work"] == "dispatch":
        return {"bytes": row + token + 4.0 * (P * (4 if case["weighted"] else 3) + 2 * case["experts"]), "flops": 0.0}
    if case["work"] == "combine":
        return {"bytes": row + token + 8.0 * P, "flops": 2.0 * P * d}
    if case["work"] == "combine_grad":
        return {"bytes": 2 * row + token + 12.0 * P, "flops": 3.0 * P * d}
    return {"bytes": row + token * (2 if case["weighted"] else 1) + (12.0 if case["weighted"] else 4.0) * P, "flops": (4.0 if case["weighted"] else 1.0) * P * d}


def _exact_rows(s):
    T, k, d, w = s["tokens"], s["top_k"], s["d"], s["weights"]
    token = torch.arange(T * k, device="cuda") // k
    w = torch.ones(T * k, dtype=torch.float64, device="cuda") if w is None else w.double().flatten()
    if s["work"] == "dispatch":
        flat = s["ids"].flatten()
        lists = [(flat == e).nonzero()[:, 0] for e in range(s["experts"])]
        perm = torch.cat(lists)
        counts = torch.tensor([len(v) for v in lists], dtype=torch.int32)
        off = torch.tensor([sum(len(v) for v in lists[:e]) for e in range(s["experts"] + 1)], dtype=torch.int32)
        slots = torch.zeros(T * k, dtype=torch.int32, device="cuda").scatter_(0, perm, torch.arange(T * k, dtype=torch.int32, device="cuda"))
        rows = torch.empty(T * k, d, dtype=torch.float64, device="cuda")
        for i in range(0, T * k, 16384):
            rows[i:i + 16384] = s["x"][token[perm[i:i + 16384]]].double() * w[perm[i:i + 16384], None]
        return {"rows": rows, "counts": counts, "off": off, "perm": perm.int(), "slots": slots}
    at = s["slots"].long().view(T, k)
    w = w.view(T, k)
    if s["work"] in ("combine", "dispatch_grad"):
        rows = s["rows"] if s["work"] == "combine" else s["drows"]
        y = torch.zeros(T, d, dtype=torch.float64, device="cuda")
        for j in range(k):
            y += w[:, j, None] * rows[at[:, j]].double()
        if s["work"] == "combine":
            return {"y": y}
        if s["weights"] is None:
            return {"dx": y}
        return {"dx": y, "dweights": torch.stack([torch.einsum("td,td->t", rows[at[:, j]].double(), s["x"].double()) for j in range(k)], 1)}
    drows = torch.empty(T * k, d, dtype=torch.float64, device="cuda")
    dy, dgates = s["dy"].double(), torch.empty(T, k, dtype=torch.float64, device="cuda")
    for j in range(k):
        drows[at[:, j]] = w[:, j, None] * dy
        dgates[:, j] = torch.einsum("td,td->t", s["rows"][at[:, j]].double(), dy)
    return {"drows": drows, "dgates": dgates}


def _exact_gate(s):
    """Through the Jacobian of the softmax over all experts, or over the picks."""
    z, at, dg = s["logits"].double(), s["ids"].long(), s["dgates"].double()
    if s["renorm"]:
        g = torch.softmax(z.gather(1, at), dim=1)
        jacobian = torch.diag_embed(g) - g[:, :, None] * g[:, None, :]
        return {"dlogits": torch.zeros_like(z).scatter_(1, at, torch.einsum("tjm,tj->tm", jacobian, dg))}
    p = torch.softmax(z, dim=1)
    picked = p.gather(1, at)
    out = torch.zeros_like(z)
    for j in range(at.shape[1]):
        out -= dg[:, j, None] * picked[:, j, None] * p
    return {"dlogits": out.scatter_add_(1, at, dg * picked)}


def _exact_lowrank(s):
    n, G = s["rows"], s["adapters"]
    if s["sorted"]:
        bounds = s["off"].tolist()
        lists = [torch.arange(bounds[g], bounds[g + 1], device="cuda") for g in range(G)]
    else:
        lists = [(s["ids"] == g).nonzero()[:, 0] for g in range(G)]
    sc = s["scales"].double()
    forward = s["work"] == "lowrank"
    out = (s["base"] if forward else s["dx_base"]).double()
    vs = torch.zeros(n, s["rank"], dtype=torch.float64, device="cuda")
    dA = torch.zeros(G, s["rank"], s["in"], dtype=torch.float64, device="cuda") if not forward else None
    dB = torch.zeros(G, s["out"], s["rank"], dtype=torch.float64, device="cuda") if not forward else None
    for g, at in enumerate(lists):
        A, B, x = s["A"][g].double(), s["B"][g].double(), s["x"][at].double()
        v = torch.einsum("nk,rk->nr", x, A)
        vs[at] = v
        if forward:
            out[at] += sc[g] * torch.einsum("nr,mr->nm", v, B)
        else:
            dy = s["dy"][at].double()
            dv = sc[g] * torch.einsum("nm,mr->nr", dy, B)
            out[at] += torch.einsum("nr,rk->nk", dv, A)
            dA[g] = torch.einsum("nr,nk->rk", dv, x)
            dB[g] = sc[g] * torch.einsum("nm,nr->mr", dy, v)
    if not forward:
        return {"dx": out, "dA": dA, "dB": dB}
    return {"y": out, "v": vs} if s["save"] else {"y": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["work"] == "gate_grad":
        return _exact_gate(s)
    return _exact_lowrank(s) if case["work"].startswith("lowrank") else _exact_rows(s)
