"""The cases by which the operators of a layer of experts held in 8 bits are measured, with their plain forms.

`run` with `own` false computes each operator from elementary torch operations in fp32, rounded once at the end;
with `own` true it makes the calls of `paper_1604_00981_b200.binding`.  The cases:

balance    the router's balance loss with the experts' counts, and its gradient
quantize   rows, or matrices in both directions, to 8 bits with a power of two as scale for each block of 128
gate       silu(gate) * up between the experts' two products, into 8 bits, with a checkpoint of its input in 8 bits
gate_back  its gradient from that checkpoint
product    the experts' products of 8-bit rows with 8-bit matrices
gradient   the gradient of the experts' matrices from the 8-bit checkpoint of their inputs
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
BLOCK = 128
LOWEST = -110                          # exponent of the smallest scale
POWER = {"e4m3": 9, "e5m2": 16}        # the largest number of each format is 0.875 * 2 ** POWER
COEFFICIENT = 0.01                     # of the balance loss in the whole loss


def listed():
    return [
        # the router of a small block, one worker's mini-batch: latency alone
        dict(name="balance_256x8_k2_f32", op="balance", dtype="f32", tokens=256, k=2, experts=8, padded=False),
        # a large batch with padding, many small experts
        dict(name="balance_32768x256_k8_bf16", op="balance", dtype="bf16", tokens=32768, k=8, experts=256, padded=True),
        # the rows of a few tokens, odd width
        dict(name="quantize_3x1001_f32", op="quantize", dtype="f32", fmt="e4m3", batch=0, rows=3, width=1001),
        # the master weights of a layer of 16 experts, for the forward and the backward pass
        dict(name="quantize_16x2816x2048_f32", op="quantize", dtype="f32", fmt="e4m3", batch=16, rows=2816, width=2048),
        # a training batch's activations, two experts to a token
        dict(name="gate_16384x1408_bf16", op="gate", dtype="bf16", fmt="e4m3", rows=16384, width=1408),
        # a ragged batch, odd width
        dict(name="gate_back_777x1000_f32", op="gate_back", dtype="f32", fmt="e4m3", rows=777, width=1000),
        dict(name="gate_back_16384x1408_bf16", op="gate_back", dtype="bf16", fmt="e4m3", rows=16384, width=1408),
        # one token and its eight experts: the weights are all there is to read
        dict(name="product_8x2816x2048_e64_bf16", op="product", dtype="bf16", fmt="e4m3", rows=8, width=2816, depth=2048, experts=64),
        # a small ragged batch in fp32, its gradient's format on one side
        dict(name="product_999x1001x500_e7_f32", op="product", dtype="f32", fmt="e5m2", rows=999, width=1001, depth=500, experts=7),
        # a training batch
        dict(name="product_16384x2816x2048_e16_bf16", op="product", dtype="bf16", fmt="e4m3", rows=16384, width=2816, depth=2048, experts=16),
        dict(name="gradient_999x500x1001_e7_f32", op="gradient", dtype="f32", fmt="e4m3", rows=999, width=500, depth=1001, experts=7),
        dict(name="gradient_16384x2816x2048_e16_bf16", op="gradient", dtype="bf16", fmt="e4m3", rows=16384, width=2816, depth=2048, experts=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _round_some(rng, n, to):
    """Half of the drawn sizes are multiples of `to`, the others what they are."""
    return max(to, n // to * to) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["balance", "quantize", "gate", "gate_back", "product", "product", "gradient", "gradient"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "balance":
        k = rng.randint(1, 8)
        experts = max(k, _log(rng, 4, 512))
        return dict(op=op, dtype=dtype, tokens=_log(rng, 1, min(32768, 32768 * 256 // experts)), k=k, experts=experts, padded=rng.random() < 0.5)
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    width = _round_some(rng, _log(rng, 48, 4096), 128)
    if op in ("gate", "gate_back"):
        return dict(op=op, dtype=dtype, fmt=fmt, rows=_log(rng, 1, min(16384, 16384 * 704 // width)), width=width)
    if op == "quantize":
        if rng.random() < 0.5:
            return dict(op=op, dtype=dtype, fmt=fmt, batch=0, rows=_log(rng, 1, min(32768, 32768 * 2048 // width)), width=width)
        rows = _round_some(rng, _log(rng, 48, 4096), 128)
        return dict(op=op, dtype=dtype, fmt=fmt, batch=_log(rng, 1, min(64, max(1, 16 * 2816 * 2048 // (rows * width)))), rows=rows, width=width)
    depth = _round_some(rng, _log(rng, 48, 4096), 128)
    most = 16384 * 2816 * 2048 // (width * depth)
    experts = _log(rng, 1, max(1, min(64, 32 * 2816 * 2048 // (width * depth))))
    return dict(op=op, dtype=dtype, fmt=fmt, rows=_log(rng, 1, min(32768, most)), width=width, depth=depth, experts=experts)


# ------------------------------------------------------------------ inputs


def _offsets(gen, rows, experts):
    """Popular and unpopular experts, one row in fifty not in use; a few rows go to experts of their own."""
    if rows <= experts:
        counts = torch.zeros(experts, dtype=torch.int64, device="cuda")
        counts[torch.randperm(experts, device="cuda", generator=gen)[:rows]] = 1
    else:
        p = torch.softmax(0.5 * torch.randn(experts, device="cuda", generator=gen), 0)
        ids = torch.multinomial(p, rows - rows // 50, replacement=True, generator=gen)
        counts = torch.bincount(ids, minlength=experts)
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()


def _rows8(gen, rows, width, fmt):
    """Rows in 8 bits and their scales, as a layer before keeps them: leading dimensions of whole 16-byte chunks, and padding."""
    x = torch.randn(rows, width, device="cuda", generator=gen) * torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=gen))
    q, scale = _plain_quantize(x, fmt)
    out = torch.zeros(rows, (width + 15) // 16 * 16, dtype=q.dtype, device="cuda")[:, :width]
    out.copy_(q)
    return out, scale


def _new8(fmt, *shape):
    pad = (shape[-1] + 15) // 16 * 16
    return torch.empty(*shape[:-1], pad, dtype=DTYPES[fmt], device="cuda")[..., : shape[-1]]


def _new_scale(*shape):
    return torch.empty(shape, dtype=torch.float8_e8m0fnu, device="cuda")


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case)
    if op == "balance":
        T, E, k = case["tokens"], case["experts"], case["k"]
        logits = torch.randn(T, E, device=dev, generator=gen) + 0.7 * torch.randn(E, device=dev, generator=gen)
        s["logits"] = logits.to(dt)
        ids = torch.topk(logits, k, dim=1).indices.to(torch.int32)
        ids[torch.rand(T, k, device=dev, generator=gen) < 0.02] = -1  # over an expert's capacity
        s["ids"] = ids.contiguous()
        s["mask"] = (torch.rand(T, device=dev, generator=gen) < 0.9).to(torch.uint8) if case["padded"] else None
        s["loss"], s["counts"] = torch.empty(1, device=dev), torch.empty(E, dtype=torch.int32, device=dev)
        s["slope"] = torch.empty(E, device=dev)
        s["grad"], s["dlogits"] = torch.full((1,), COEFFICIENT, device=dev), torch.empty(T, E, dtype=dt, device=dev)
    elif op == "quantize":
        B, R, D, fmt = case["batch"], case["rows"], case["width"], case["fmt"]
        if B == 0:
            x = torch.randn(R, D, device=dev, generator=gen) * torch.exp(torch.randn(R, 1, device=dev, generator=gen))
            s["x"], s["q"], s["scale"] = x.to(dt), _new8(fmt, R, D), _new_scale(R, _blocks(D))
        else:
            s["x"] = (torch.randn(B, R, D, device=dev, generator=gen) * D ** -0.5).to(dt)
            s["q"], s["qt"], s["scale"] = _new8(fmt, B, R, D), _new8(fmt, B, D, R), _new_scale(B, _blocks(R), _blocks(D))
    elif op in ("gate", "gate_back"):
        R, F, fmt = case["rows"], case["width"], case["fmt"]
        h = torch.randn(R, 2 * F, device=dev, generator=gen) * torch.exp(0.3 * torch.randn(R, 1, device=dev, generator=gen))
        if op == "gate":
            s["h"] = h.to(dt)
            s["a"], s["a_scale"] = _new8(fmt, R, F), _new_scale(R, _blocks(F))
            s["h8"], s["h_scale"] = _new8(fmt, R, 2, F), _new_scale(R, 2, _blocks(F))
        else:
            q, s["h_scale"] = _plain_quantize(h.view(R, 2, F), fmt)
            s["h8"] = _new8(fmt, R, 2, F)
            s["h8"].copy_(q)
            s["da"] = (0.1 * torch.randn(R, F, device=dev, generator=gen)).to(dt)
            s["dh"] = torch.empty(R, 2 * F, dtype=dt, device=dev)
    else:
        S, N, K, E, fmt = case["rows"], case["width"], case["depth"], case["experts"], case["fmt"]
        s["offsets"] = _offsets(gen, S, E)
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
        s["x"], s["x_scale"] = _rows8(gen, S, K, fmt)
        if op == "product":
            w = _new8("e4m3", E, N, K)
            s["w"], s["w_scale"] = w, _new_scale(E, _blocks(N), _blocks(K))
            for e in range(E):  # one at a time: the matrices in fp32 are four times as large
                q, scale = _plain_quantize_matrices(torch.randn(1, N, K, device=dev, generator=gen) * K ** -0.5, "e4m3")
                w[e].copy_(q[0])
                s["w_scale"][e].copy_(scale[0])
            s["y"] = torch.empty(S, N, dtype=dt, device=dev)
        else:
            s["dy"] = (0.1 * torch.randn(S, N, device=dev, generator=gen)).to(dt)
            s["dw"] = torch.empty(E, N, K, dtype=dt, device=dev)
    return s


# ------------------------------------------------------------------ plain forms


def _exponent(x, fmt):
    """The smallest e with max|x| <= largest * 2 ** e over the last dimension, infinities and NaN apart."""
    a = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(a)
    e = torch.where(a > 0, e - POWER[fmt] + (m > 0.875), 0)
    return e.clamp(min=LOWEST)


def _pad(x, dim):
    n = x.shape[dim]
    more = list(x.shape)
    more[dim] = _blocks(n) * BLOCK - n
    return torch.cat([x, x.new_zeros(more)], dim) if more[dim] else x


def _scale8(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _plain_quantize(x, fmt):
    """x [..., width] fp32 -> values in 8 bits of the same shape, scales [..., blocks]."""
    b = _pad(x, -1).unflatten(-1, (-1, BLOCK))
    e = _exponent(b, fmt)
    q = torch.ldexp(b, -e[..., None])
    q = torch.where(torch.isfinite(q), q, torch.nan).to(DTYPES[fmt])
    return q.flatten(-2)[..., : x.shape[-1]], _scale8(e)


def _plain_quantize_matrices(w, fmt):
    """w [batch, rows, cols] fp32 -> values in 8 bits, scales [batch, blocks of rows, blocks of columns]."""
    b = _pad(_pad(w, -1), -2).unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, BLOCK)).transpose(-3, -2)
    e = _exponent(b.flatten(-2), fmt)
    q = torch.ldexp(b, -e[..., None, None])
    q = torch.where(torch.isfinite(q), q, torch.nan).to(DTYPES[fmt]).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    return q[..., : w.shape[-2], : w.shape[-1]], _scale8(e)


def _wide(q, scale, dtype=torch.float32):
    """What 8-bit values and the scales of their blocks of 128 stand for."""
    return q.to(dtype) * scale.to(dtype).repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]


def _wide_matrices(q, scale, dtype=torch.float32):
    return _wide(q, scale.to(dtype).repeat_interleave(BLOCK, -2)[..., : q.shape[-2], :], dtype)


def _by_expert(rows, offsets, most):
    """rows [S, D] -> [experts, most, D], zero where an expert has fewer."""
    at = offsets[:-1, None].long() + torch.arange(most, device=rows.device)
    there = at < offsets[1:, None]
    return torch.where(there[..., None], rows[torch.where(there, at, 0)], 0.0)


def _plain(s):
    op, dt = s["op"], DTYPES[s["dtype"]]
    if op == "balance":
        T, E, k = s["tokens"], s["experts"], s["k"]
        x = s["logits"].float()
        counted = torch.ones(T, device="cuda") if s["mask"] is None else (s["mask"] != 0).float()
        top = x.amax(1)
        top = torch.where(torch.isneginf(top), 0.0, top)
        z = torch.exp(x - top[:, None])
        total = z.sum(1)
        p = torch.where(total[:, None] > 0, z / total[:, None], 0.0)
        p = torch.where(counted[:, None] > 0, p, 0.0)
        n = counted.sum()
        ids = torch.where(counted[:, None] > 0, s["ids"].long(), -1).reshape(-1)
        ids = torch.where((ids >= 0) & (ids < E), ids, E)
        counts = torch.bincount(ids, minlength=E + 1)[:E]
        slope = torch.where(n > 0, E * counts / (n * n * k), 0.0)
        loss = (slope * p.sum(0)).sum()
        dlogits = s["grad"] * p * (slope - (p * slope).sum(1, keepdim=True))
        return [loss.reshape(1), counts.int(), dlogits.to(dt)]
    if op == "quantize":
        if s["batch"] == 0:
            return list(_plain_quantize(s["x"].float(), s["fmt"]))
        q, scale = _plain_quantize_matrices(s["x"].float(), s["fmt"])
        return [q, q.view(torch.uint8).transpose(-2, -1).contiguous().view(q.dtype), scale]
    if op == "gate":
        h = s["h"].float().view(s["rows"], 2, s["width"])
        a = h[:, 0] / (1.0 + torch.exp(-h[:, 0])) * h[:, 1]
        return [*_plain_quantize(a, s["fmt"]), *_plain_quantize(h, s["fmt"])]
    if op == "gate_back":
        h, da = _wide(s["h8"], s["h_scale"]), s["da"].float()
        g, u = h[:, 0], h[:, 1]
        sig = 1.0 / (1.0 + torch.exp(-g))
        return [torch.cat([da * u * sig * (1.0 + g * (1.0 - sig)), da * g * sig], 1).to(dt)]
    offsets, most = s["offsets"], s["most"]
    x = _by_expert(_wide(s["x"], s["x_scale"]), offsets, most)
    if op == "gradient":
        return [(_by_expert(s["dy"].float(), offsets, most).transpose(1, 2) @ x).to(dt)]
    y = x @ _wide_matrices(s["w"], s["w_scale"]).transpose(1, 2)
    row = torch.arange(s["rows"], device="cuda")
    e = (row[:, None] >= offsets[None, 1:]).sum(1)
    used = e < s["experts"]
    e = torch.where(used, e, 0)
    return [torch.where(used[:, None], y[e, torch.where(used, row - offsets[e], 0)], 0.0).to(dt)]


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    from paper_1604_00981_b200 import binding as sgdb

    op = s["op"]
    if op in ("balance", "gradient") and "workspace" not in s:  # kept from pass to pass, as a training loop does
        if op == "balance":
            need = sgdb.sgdb_balance_loss_workspace_bytes(s["tokens"], s["experts"])
        else:
            need = sgdb.sgdb_experts_gradient_workspace_bytes(s["rows"], s["width"], s["depth"], s["experts"])
        s["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    if op == "balance":
        sgdb.sgdb_balance_loss(s["logits"], s["ids"], s["mask"], s["loss"], s["counts"], s["slope"], s["workspace"])
        sgdb.sgdb_balance_loss_backward(s["grad"], s["logits"], s["mask"], s["slope"], s["dlogits"])
        return [s["loss"], s["counts"], s["dlogits"]]
    if op == "quantize":
        if s["batch"] == 0:
            sgdb.sgdb_quantize(s["x"], s["q"], s["scale"])
            return [s["q"], s["scale"]]
        sgdb.sgdb_quantize_matrices(s["x"], s["q"], s["qt"], s["scale"])
        return [s["q"], s["qt"], s["scale"]]
    if op == "gate":
        sgdb.sgdb_gate(s["h"], s["a"], s["a_scale"], s["h8"], s["h_scale"])
        return [s["a"], s["a_scale"], s["h8"], s["h_scale"]]
    if op == "gate_back":
        sgdb.sgdb_gate_backward(s["da"], s["h8"], s["h_scale"], s["dh"])
        return [s["dh"]]
    if op == "product":
        sgdb.sgdb_experts_product(s["x"], s["x_scale"], s["w"], s["w_scale"], s["offsets"], s["y"])
        return [s["y"]]
    sgdb.sgdb_experts_gradient(s["dy"], s["x"], s["x_scale"], s["offsets"], s["dw"], s["workspace"])
    return [s["dw"]]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "balance":
        T, E, k = case["tokens"], case["experts"], case["k"]
        return {"bytes": 2 * T * E * size + 4 * T * k + 4 * E, "flops": 12 * T * E}
    if op == "quantize":
        R, D, B = case["rows"], case["width"], case["batch"]
        if B == 0:
            return {"bytes": R * D * (size + 1) + R * _blocks(D), "flops": 2 * R * D}
        return {"bytes": B * R * D * (size + 2) + B * _blocks(R) * _blocks(D), "flops": 2 * B * R * D}
    if op == "gate":
        R, F = case["rows"], case["width"]
        return {"bytes": R * F * (2 * size + 3) + 3 * R * _blocks(F), "flops": 12 * R * F}
    if op == "gate_back":
        R, F = case["rows"], case["width"]
        return {"bytes": R * F * (3 * size + 2) + 2 * R * _blocks(F), "flops": 15 * R * F}
    S, N, K, E = case["rows"], case["width"], case["depth"], case["experts"]
    used = S if S <= E else S - S // 50
    rows = used * (K + _blocks(K) + N * size)
    if op == "product":
        return {"bytes": rows + min(S, E) * N * K, "flops": 2 * used * N * K}
    return {"bytes": rows + E * N * K * size, "flops": 2 * used * N * K}


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_scale(x, fmt):
    """The power of two that takes the largest magnitude of each row of x to at most the format's largest number."""
    top = x.abs().max(-1, keepdim=True).values
    most = float(torch.finfo(DTYPES[fmt]).max)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / most)), 0.0)
    return torch.exp2(e.clamp(min=LOWEST))


def _exact_scaled(x, fmt):
    """x [rows, width] over the scales of its blocks, not rounded."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        piece = x[:, c : c + BLOCK]
        out[:, c : c + BLOCK] = piece / _exact_scale(piece, fmt)
    return out


def _exact_silu(g):
    return g * torch.special.expit(g)


def exact(case, seed):
    s = prepare(case, seed)
    op, fmt = case["op"], case.get("fmt")
    if op == "balance":
        T, E, k = case["tokens"], case["experts"], case["k"]
        kept = torch.arange(T, device="cuda") if s["mask"] is None else s["mask"].nonzero()[:, 0]
        p = torch.softmax(s["logits"].double()[kept], 1)
        counts = torch.stack([(s["ids"][kept] == e).sum() for e in range(E)])
        n = len(kept)
        if n == 0:
            return [torch.zeros(1, dtype=torch.float64), counts.int(), torch.zeros(T, E, dtype=torch.float64, device="cuda")]
        share = counts.double() / (n * k)
        loss = E * torch.dot(share, p.mean(0))
        dlogits = torch.zeros(T, E, dtype=torch.float64, device="cuda")
        dp = float(s["grad"]) * E * share / n
        dlogits[kept] = p * (dp - (p @ dp)[:, None])
        return [loss.reshape(1), counts.int(), dlogits]
    if op == "quantize":
        x = s["x"].double()
        if case["batch"] == 0:
            return [_exact_scaled(x, fmt), None]
        out = torch.empty_like(x)
        for r in range(0, case["rows"], BLOCK):
            for c in range(0, case["width"], BLOCK):
                piece = x[:, r : r + BLOCK, c : c + BLOCK]
                out[:, r : r + BLOCK, c : c + BLOCK] = piece / _exact_scale(piece.reshape(len(piece), -1), fmt)[..., None]
        return [out, out.mT, None]
    if op == "gate":
        h = s["h"].double()
        g, u = h.chunk(2, 1)
        h8 = torch.stack([_exact_scaled(g.contiguous(), fmt), _exact_scaled(u.contiguous(), fmt)], 1)
        return [_exact_scaled(_exact_silu(g) * u, fmt), None, h8, None]
    if op == "gate_back":
        h = s["h8"].double()
        for b in range(_blocks(case["width"])):
            h[..., b * BLOCK : (b + 1) * BLOCK] *= s["h_scale"][..., b].double()[..., None]
        with torch.enable_grad():
            g, u = h[:, 0].clone().requires_grad_(), h[:, 1].clone().requires_grad_()
            dg, du = torch.autograd.grad(_exact_silu(g) * u, (g, u), s["da"].double())
        return [torch.cat([dg, du], 1)]
    S, N, K, E = case["rows"], case["width"], case["depth"], case["experts"]
    edges = s["offsets"].tolist()
    x = s["x"].double()
    for b in range(_blocks(K)):
        x[:, b * BLOCK : (b + 1) * BLOCK] *= s["x_scale"][:, b : b + 1].double()
    if op == "gradient":
        return [torch.stack([s["dy"][a:b].double().mT @ x[a:b] for a, b in zip(edges, edges[1:])])]
    y = torch.zeros(S, N, dtype=torch.float64, device="cuda")
    for e, (a, b) in enumerate(zip(edges, edges[1:])):
        if b > a:
            scale = s["w_scale"][e].double()
            w = s["w"][e].double() * torch.kron(scale, torch.ones(BLOCK, BLOCK, dtype=torch.float64, device="cuda"))[:N, :K]
            y[a:b] = torch.nn.functional.linear(x[a:b], w)
    return [y]
