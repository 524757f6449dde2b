"""The operators around the experts of an MoE layer, as cases that can be timed and compared: tokens sorted by expert
and dispatched to rows, rows combined back with their weights, the norms before and after the block with its gate and
residual scale, and the gradients of all of these and of the gate.

A case is a dict of plain values:
  op              "dispatch"       expert ids -> row order, rows of the tokens in that order
                  "dispatch_grad"  gradient of the rows -> gradient of the tokens
                  "combine"        rows and weights -> tokens
                  "combine_grad"   gradient of the tokens -> gradients of the rows, the weights and the gate's logits
                  "before"         residual stream and its update -> new residual stream, the block's normed input
                  "before_grad"    gradients of both -> gradients of residual stream, update and norm parameters
                  "after"          residual stream and the block's output -> residual + scale * gate * norm(output)
                  "after_grad"     its gradient -> gradients of the output, the norm parameters and the gate
  T, H, dtype     tokens, embedding size, type of the rows ("bf16", "fp16", "fp32")
  E, k            experts, experts per token                                          (dispatch and combine)
  zipf            > 0: expert popularity (e + 1)^-zipf is added to the gate logits    (dispatch and combine)
  padded          share of the tokens, at the end of the batch, that have no expert   (dispatch and combine)
  norm            "rms" or "layer" (the latter with a bias)                           (before and after)
  gate            "none", "channel" [H], "token" [T] or "full" [T,H]                  (after)
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EPS = 1e-5
_SCALE = 0.5          # of the block's output where it enters the residual stream
_GATES = ("none", "channel", "token", "full")

# Layers of workloads.py: (H, E, k)
_SHAPES = {
    "tiny": (256, 4, 2),
    "mixtral": (4096, 8, 2),
    "qwen2": (3584, 64, 8),
    "qwen2_table2": (2048, 64, 4),
    "phi35": (4096, 16, 2),
}
_ROW_BYTES = 32768 * 2 * 4096 * 2       # rows of the largest dispatch or combine
_STREAM_BYTES = 16384 * 4096 * 2        # residual stream of the largest norm


def _moved(op, T, H, E, k, dtype="bf16", zipf=0.0, padded=0.0, name=None):
    c = dict(op=op, T=T, H=H, E=E, k=k, dtype=dtype, zipf=zipf, padded=padded)
    if name is not None:
        c["name"] = name
    return c


def _normed(op, T, H, dtype="bf16", norm="rms", gate="none", name=None):
    c = dict(op=op, T=T, H=H, dtype=dtype, norm=norm)
    if op.startswith("after"):
        c["gate"] = gate
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence decoding: the residual stream of one token, where only latency counts
        _normed("before", 1, 4096, name="before_1_mixtral"),
        # a small decode batch whose experts are the caller's own
        _moved("dispatch", 16, 4096, 8, 2, name="dispatch_16_mixtral"),
        # a decode batch over many small experts
        _moved("combine", 48, 3584, 64, 8, name="combine_48_qwen2"),
        # the smallest training step, in single precision, of which a quarter is padding
        _moved("combine_grad", 128, 256, 4, 2, dtype="fp32", padded=0.25, name="combine_grad_128_tiny_fp32"),
        # a chunk of a prompt, rows that are not a multiple of 16 bytes, a gate for each token, mean and bias
        _normed("after", 509, 4097, dtype="fp16", norm="layer", gate="token", name="after_509_odd_fp16"),
        # training on a short ragged batch, rows of an odd length
        _moved("dispatch_grad", 2047, 1001, 16, 2, dtype="fp16", padded=0.1, name="dispatch_grad_2047_odd_fp16"),
        # prefill over many small experts
        _moved("dispatch", 8192, 2048, 64, 4, name="dispatch_8192_qwen2_table2"),
        # training: the norm between attention and the block
        _normed("before_grad", 4096, 3584, name="before_grad_4096_qwen2"),
        # the benchmark's batch: the residual stream enters the block
        _normed("before", 8192, 4096, name="before_8192_mixtral"),
        # prefill, the popularity of the experts uneven
        _moved("combine", 16384, 4096, 16, 2, zipf=1.2, name="combine_16384_phi35"),
        # training: what leaves the block, a gate for each channel
        _normed("after_grad", 16384, 4096, gate="channel", name="after_grad_16384_phi35"),
        # training on the largest batch, experts uneven
        _moved("combine_grad", 32768, 4096, 8, 2, zipf=1.2, name="combine_grad_32768_skewed"),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any operator, any number of tokens up to the largest (even over the logarithm), the widths of the
    layers or any other one, the usual options more often than the others."""
    op = rng.choice(("dispatch", "dispatch_grad", "combine", "combine_grad", "before", "before_grad", "after", "after_grad"))
    H, E, k = _SHAPES[rng.choice(sorted(_SHAPES))]
    if rng.random() < 0.4:
        H = _log_uniform(rng, 33, 8192)
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp16", "fp32"))
    row = H * _DTYPES[dtype].itemsize
    if op in ("before", "before_grad", "after", "after_grad"):
        T = _log_uniform(rng, 1, min(32768, _STREAM_BYTES // row))
        return _normed(op, T, H, dtype, rng.choice(("rms", "rms", "layer")), rng.choice(_GATES))
    if rng.random() < 0.4:
        E = _log_uniform(rng, 2, 256)
        k = rng.randint(1, min(E, 8))
    T = _log_uniform(rng, 1, min(32768, _ROW_BYTES // (row * k)))
    return _moved(op, T, H, E, k, dtype, rng.choice((0.0, 0.0, 1.2)), rng.choice((0.0, 0.0, 0.25)))


class _State:
    pass


def _normal(g, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _stream(g, T, H, dtype):
    """Rows of a residual stream: a few channels are much larger than the others."""
    v = torch.empty((T, H), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)
    v[:, torch.randint(0, H, (1 + H // 512,), device="cuda", generator=g)] *= 12.0
    return v.to(dtype)


def prepare(case, seed):
    """The tensors a program has before the call, and the ones the results go to."""
    s = _State()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s.op, T, H, dtype = case["op"], case["T"], case["H"], _DTYPES[case["dtype"]]
    s.workspace = None
    new = lambda shape, dt=dtype: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    if "E" in case:
        E, k = case["E"], case["k"]
        R = T * k
        s.E, s.k = E, k
        logits = _normal(g, (T, E), torch.float32)
        if case["zipf"] > 0:
            logits += torch.log(torch.arange(1, E + 1, dtype=torch.float32, device="cuda") ** -case["zipf"])
        top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
        s.w = torch.softmax(top[:, :k], dim=1).contiguous()
        s.ids = ids[:, :k].to(torch.int32).contiguous()
        if case["padded"] > 0:
            s.ids[T - int(T * case["padded"]):] = -1
        if s.op == "dispatch":
            s.x = _stream(g, T, H, dtype)
            s.offsets, s.perm, s.inv = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in ((E + 1,), (R,), (T, k)))
            s.rows = new((R, H))
            return s
        key = torch.where(s.ids.reshape(-1) < 0, E, s.ids.reshape(-1))
        order = torch.argsort(key, stable=True)
        inv = torch.empty(R, dtype=torch.int32, device="cuda")
        inv[order] = torch.arange(R, dtype=torch.int32, device="cuda")
        s.inv = torch.where(key == E, -1, inv).to(torch.int32).reshape(T, k)
        s.rows = _normal(g, (R, H), dtype)
        if s.op == "combine_grad":
            s.g = _normal(g, (T, H), dtype)
            s.grad_rows, s.grad_w, s.grad_logits = new((R, H)), new((T, k), torch.float32), new((T, E), torch.float32)
        else:
            s.out = new((T, H))
        return s
    s.norm, s.gate_kind = case["norm"], case.get("gate", "none")
    s.gamma = _normal(g, (H,), dtype, 0.1, 1.0)
    s.beta = _normal(g, (H,), dtype, 0.1) if s.norm == "layer" else None
    f32 = torch.float32
    if s.op == "before":
        s.residual, s.update = _stream(g, T, H, dtype), _normal(g, (T, H), dtype)
        s.sum, s.x = new((T, H)), new((T, H))
    elif s.op == "before_grad":
        s.sum, s.gx, s.gs = _stream(g, T, H, dtype), _normal(g, (T, H), dtype), _normal(g, (T, H), dtype)
        s.grad_residual, s.grad_update = new((T, H)), new((T, H))
        s.grad_gamma, s.grad_beta = new((H,), f32), new((H,), f32) if s.beta is not None else None
    else:
        s.y = _normal(g, (T, H), dtype, 3.0, 0.5)
        s.gate = {"none": lambda: None, "channel": lambda: _normal(g, (H,), dtype, 0.3, 0.5),
                  "token": lambda: torch.sigmoid(_normal(g, (T,), f32)), "full": lambda: _normal(g, (T, H), dtype, 0.3, 0.5)}[s.gate_kind]()
        if s.op == "after":
            s.residual, s.out = _stream(g, T, H, dtype), new((T, H))
        else:
            s.g, s.grad_y = _normal(g, (T, H), dtype), new((T, H))
            s.grad_gamma, s.grad_beta = new((H,), f32), new((H,), f32) if s.beta is not None else None
            s.grad_gate = None if s.gate is None else new(tuple(s.gate.shape), dtype if s.gate_kind == "full" else f32)
    return s


def _own(s):
    """The calls of the framework."""
    import paper_2502_19811_amd as moe
    if s.op == "dispatch":
        if s.workspace is None:
            s.workspace = torch.empty(moe.moe_sort_workspace_bytes(s.ids.shape[0], s.E, s.k), dtype=torch.uint8, device="cuda")
        moe.moe_sort_tokens(s.ids, s.E, s.offsets, s.perm, s.inv, s.workspace)
        moe.moe_dispatch(s.x, s.inv, s.rows)
        return {"offsets": s.offsets, "perm": s.perm, "inv": s.inv, "rows": s.rows}
    if s.op == "dispatch_grad":
        moe.moe_dispatch_backward(s.rows, s.inv, s.out)
        return {"grad_x": s.out}
    if s.op == "combine":
        moe.moe_combine(s.rows, s.inv, s.w, s.out)
        return {"out": s.out}
    if s.op == "combine_grad":
        moe.moe_combine_backward(s.g, s.rows, s.inv, s.w, s.grad_rows, s.grad_w)
        moe.moe_route_topk_backward(s.ids, s.w, s.grad_w, s.grad_logits)
        return {"grad_rows": s.grad_rows, "grad_weights": s.grad_w, "grad_logits": s.grad_logits}
    norm = moe.MOE_NORM_RMS if s.norm == "rms" else moe.MOE_NORM_LAYER
    if s.op == "before":
        moe.moe_norm_before(s.residual, s.update, _SCALE, s.gamma, s.beta, norm, _EPS, s.sum, s.x)
        return {"sum": s.sum, "x": s.x}
    gate_kind = (moe.MOE_GATE_NONE, moe.MOE_GATE_CHANNEL, moe.MOE_GATE_TOKEN, moe.MOE_GATE_FULL)[_GATES.index(s.gate_kind)]
    if s.op == "after":
        moe.moe_norm_after(s.residual, s.y, s.gamma, s.beta, s.gate, gate_kind, _SCALE, norm, _EPS, s.out)
        return {"out": s.out}
    if s.workspace is None:
        s.workspace = torch.empty(moe.moe_norm_workspace_bytes(*s.grad_y.shape) if s.op == "after_grad"
                                  else moe.moe_norm_workspace_bytes(*s.sum.shape), dtype=torch.uint8, device="cuda")
    if s.op == "before_grad":
        moe.moe_norm_before_backward(s.sum, s.gamma, s.gx, s.gs, _SCALE, norm, _EPS, s.grad_residual, s.grad_update,
                                     s.grad_gamma, s.grad_beta, s.workspace)
        return {"grad_residual": s.grad_residual, "grad_update": s.grad_update, "grad_gamma": s.grad_gamma, "grad_beta": s.grad_beta}
    moe.moe_norm_after_backward(s.y, s.gamma, s.beta, s.gate, gate_kind, _SCALE, s.g, norm, _EPS, s.grad_y, s.grad_gamma,
                                s.grad_beta, s.grad_gate, s.workspace)
    return {"grad_y": s.grad_y, "grad_gamma": s.grad_gamma, "grad_beta": s.grad_beta, "grad_gate": s.grad_gate}


def _n(v, norm):
    """Normed rows and the reciprocal of what they were divided by."""
    if norm == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    r = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + _EPS)
    return v * r, r


def _norm_grad(d, n, r, norm):
    """Gradient of the rows that were normed to n, from the gradient d of n."""
    d = d - n * (d * n).mean(dim=1, keepdim=True) if norm == "rms" else d - d.mean(dim=1, keepdim=True) - n * (d * n).mean(dim=1, keepdim=True)
    return r * d


def _plain(s):
    """The operators in elementary torch operations, in 32 bits."""
    if s.op == "dispatch":
        T, k = s.ids.shape
        key = s.ids.reshape(-1).long()
        key = torch.where((key < 0) | (key >= s.E), s.E, key)
        order = torch.argsort(key, stable=True)
        dropped = key[order] == s.E
        offsets = torch.cumsum((key[:, None] == torch.arange(-1, s.E, device="cuda")).sum(dim=0), dim=0).to(torch.int32)
        inv = torch.empty_like(order)
        inv[order] = torch.arange(T * k, device="cuda")
        inv = torch.where(key == s.E, -1, inv).to(torch.int32).reshape(T, k)
        rows = torch.where(dropped[:, None], s.rows, s.x[order // k])
        return {"offsets": offsets, "perm": torch.where(dropped, -1, order).to(torch.int32), "inv": inv, "rows": rows}
    if s.op in ("dispatch_grad", "combine"):
        kept = (s.inv >= 0)[:, :, None]
        v = torch.where(kept, s.rows[s.inv.clamp(min=0).long()].float(), 0.0)
        if s.op == "combine":
            v = v * s.w[:, :, None]
        return {"out" if s.op == "combine" else "grad_x": v.sum(dim=1).to(s.rows.dtype)}
    if s.op == "combine_grad":
        T, k = s.inv.shape
        kept = s.inv >= 0
        at = s.inv.clamp(min=0).long()
        g = s.g.float()[:, None, :]
        gw = torch.where(kept, (s.rows[at].float() * g).sum(dim=2), 0.0)
        grad_rows = torch.cat([s.grad_rows, s.grad_rows[:1]])      # one row more, for what the dropped slots would have
        grad_rows[torch.where(kept, at, T * k).reshape(-1)] = (s.w[:, :, None] * g).to(s.g.dtype).reshape(T * k, -1)
        d = s.w * (gw - (s.w * gw).sum(dim=1, keepdim=True))
        hot = s.ids[:, :, None] == torch.arange(s.E, device="cuda")
        return {"grad_rows": grad_rows[:-1], "grad_weights": gw, "grad_logits": torch.where(hot, d[:, :, None], 0.0).sum(dim=1)}
    gamma = s.gamma.float()
    beta = 0.0 if s.beta is None else s.beta.float()
    if s.op == "before":
        v = s.residual.float() + _SCALE * s.update.float()
        return {"sum": v.to(s.x.dtype), "x": (_n(v, s.norm)[0] * gamma + beta).to(s.x.dtype)}
    if s.op == "before_grad":
        n, r = _n(s.sum.float(), s.norm)
        gx = s.gx.float()
        total = s.gs.float() + _norm_grad(gx * gamma, n, r, s.norm)
        return {"grad_residual": total.to(s.gx.dtype), "grad_update": (_SCALE * total).to(s.gx.dtype),
                "grad_gamma": (gx * n).sum(dim=0), "grad_beta": None if s.beta is None else gx.sum(dim=0)}
    gate = 1.0 if s.gate is None else s.gate.float()[:, None] if s.gate_kind == "token" else s.gate.float()
    n, r = _n(s.y.float(), s.norm)
    if s.op == "after":
        return {"out": (s.residual.float() + _SCALE * gate * (n * gamma + beta)).to(s.out.dtype)}
    g = _SCALE * s.g.float()
    d0 = g * gate
    gg = None
    if s.gate is not None:
        gg = g * (n * gamma + beta)
        gg = gg.sum(dim=0) if s.gate_kind == "channel" else gg.sum(dim=1) if s.gate_kind == "token" else gg.to(s.g.dtype)
    return {"grad_y": _norm_grad(d0 * gamma, n, r, s.norm).to(s.g.dtype), "grad_gamma": (d0 * n).sum(dim=0),
            "grad_beta": None if s.beta is None else d0.sum(dim=0), "grad_gate": gg}


def run(s):
    """One pass, on the current stream."""
    return _own(s) if own else _plain(s)


def work(case):
    """Every input read once and every output written once."""
    op, T, H = case["op"], case["T"], case["H"]
    b = _DTYPES[case["dtype"]].itemsize
    if "E" in case:
        E, k = case["E"], case["k"]
        tokens = T - int(T * case["padded"]) if case["padded"] > 0 else T
        slots = T * k
        rows = tokens * k * H * b
        if op == "dispatch":
            return {"bytes": 4 * slots + tokens * H * b + 8 * slots + 4 * (E + 1) + rows, "flops": 0}
        if op == "dispatch_grad":
            return {"bytes": 4 * slots + rows + T * H * b, "flops": tokens * k * H}
        if op == "combine":
            return {"bytes": 8 * slots + rows + T * H * b, "flops": 2 * tokens * k * H}
        return {"bytes": 8 * slots + tokens * H * b + 2 * rows + 4 * slots + 4 * slots + 4 * T * E, "flops": 3 * tokens * k * H}
    params = H * b * (2 if case["norm"] == "layer" else 1)
    if op == "before":
        return {"bytes": 4 * T * H * b + params, "flops": 6 * T * H}
    if op == "before_grad":
        return {"bytes": 5 * T * H * b + H * b + 4 * H * (2 if case["norm"] == "layer" else 1), "flops": 15 * T * H}
    gate = {"none": 0, "channel": H * b, "token": 4 * T, "full": T * H * b}[case["gate"]]
    if op == "after":
        return {"bytes": 3 * T * H * b + params + gate, "flops": 7 * T * H}
    grads = 4 * H * (2 if case["norm"] == "layer" else 1) + {"none": 0, "channel": 4 * H, "token": 4 * T, "full": T * H * b}[case["gate"]]
    return {"bytes": 3 * T * H * b + params + gate + grads, "flops": 15 * T * H}


def exact(case, seed):
    """The definitions in 64 bits, some tokens at a time."""
    s = prepare(case, seed)
    T = case["T"]
    step = max(1, (1 << 26) // (case["H"] * case.get("k", 1)))
    parts = [slice(a, min(T, a + step)) for a in range(0, T, step)]
    D = torch.float64
    if s.op == "dispatch":
        # a slot's place: the kept slots of lower experts, and those of its own expert before it
        flat = s.ids.reshape(-1)
        rows = s.rows.to(D)
        at = 0
        for e in range(s.E):
            q = torch.nonzero(flat == e).reshape(-1)
            rows[at:at + len(q)] = s.x[q // s.k].to(D)
            at += len(q)
        return {"offsets": None, "perm": None, "inv": None, "rows": rows}
    if s.op in ("dispatch_grad", "combine"):
        out = torch.zeros((T, case["H"]), dtype=D, device="cuda")
        for p in parts:
            for j in range(s.k):
                kept = s.inv[p, j] >= 0
                w = s.w[p, j].to(D)[kept] if s.op == "combine" else torch.ones(int(kept.sum()), dtype=D, device="cuda")
                out[p][kept] += w[:, None] * s.rows[s.inv[p, j][kept].long()].to(D)
        return {"out" if s.op == "combine" else "grad_x": out}
    if s.op == "combine_grad":
        grad_rows = s.grad_rows.to(D)
        gw = torch.zeros((T, s.k), dtype=D, device="cuda")
        for p in parts:
            for j in range(s.k):
                kept = s.inv[p, j] >= 0
                at = s.inv[p, j][kept].long()
                g = s.g[p][kept].to(D)
                grad_rows[at] = s.w[p, j][kept].to(D)[:, None] * g
                gw[p, j] = gw[p, j].masked_scatter(kept, (g * s.rows[at].to(D)).sum(dim=1))
        w = s.w.to(D)
        # d w_i / d logit_j = w_i (delta_ij - w_j)
        jacobian = torch.diag_embed(w) - w[:, :, None] * w[:, None, :]
        d = (gw[:, :, None] * jacobian).sum(dim=1)
        grad_logits = torch.zeros((T, s.E + 1), dtype=D, device="cuda")
        grad_logits.scatter_add_(1, torch.where(s.ids < 0, s.E, s.ids).long(), d)
        return {"grad_rows": grad_rows, "grad_weights": gw, "grad_logits": grad_logits[:, :-1]}
    gamma, H = s.gamma.to(D), case["H"]
    beta = torch.zeros_like(gamma) if s.beta is None else s.beta.to(D)
    centred = s.norm == "layer"
    total = {}

    def note(name, p, v):
        total.setdefault(name, torch.empty((T, *v.shape[1:]), dtype=D, device="cuda"))[p] = v

    def add(name, v):
        total[name] = total[name] + v if name in total else v

    for p in parts:
        v = s.residual[p].to(D) + _SCALE * s.update[p].to(D) if s.op == "before" else (s.sum if s.op == "before_grad" else s.y)[p].to(D)
        if s.op == "before":
            note("sum", p, v)
        mean = v.sum(dim=1, keepdim=True) / H if centred else 0.0
        std = torch.sqrt(((v - mean) ** 2).sum(dim=1, keepdim=True) / H + _EPS)
        n = (v - mean) / std
        if s.op == "before":
            note("x", p, n * gamma + beta)
            continue
        if s.op == "before_grad":
            d0 = s.gx[p].to(D)
        else:
            gate = torch.ones((), dtype=D, device="cuda")
            if s.gate is not None:
                gate = s.gate.to(D) if s.gate_kind == "channel" else s.gate[p].to(D).reshape(n.shape[0], -1)
            if s.op == "after":
                note("out", p, s.residual[p].to(D) + _SCALE * gate * (n * gamma + beta))
                continue
            g = _SCALE * s.g[p].to(D)
            d0 = g * gate
            if s.gate is not None:
                gg = g * (n * gamma + beta)
                if s.gate_kind == "channel":
                    add("grad_gate", gg.sum(dim=0))
                else:
                    note("grad_gate", p, gg if s.gate_kind == "full" else gg.sum(dim=1))
        add("grad_gamma", (d0 * n).sum(dim=0))
        if s.beta is not None:
            add("grad_beta", d0.sum(dim=0))
        # n_h depends on v_i through itself, the mean and the deviation: dn_h/dv_i = (delta_hi - [1/H] - n_h n_i / H) / std
        d = d0 * gamma
        dv = d / std - n * (d * n).sum(dim=1, keepdim=True) / (H * std)
        if centred:
            dv = dv - d.sum(dim=1, keepdim=True) / (H * std)
        if s.op == "before_grad":
            dv = dv + s.gs[p].to(D)
            note("grad_residual", p, dv)
            note("grad_update", p, _SCALE * dv)
        else:
            note("grad_y", p, dv)
    return total
