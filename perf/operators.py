"""The cases by which the operators for language models are measured, with their plain forms.

`run` with `own` false computes each operator from elementary torch operations in fp32, rounded once at the end;
with `own` true it makes the calls of `paper_1604_00981_b200.binding`.  The cases:

orthogonalize    the Newton-Schulz products of an orthogonalised update, on a batch of matrices
step             one iteration of the parameter server with that update: first N of N+b gradients, mean, momentum
layer_norm       forward pass of a worker's layer norm
layer_norm_back  its backward pass with the reduction of the weights' gradients
dispatch         tokens sorted by expert and copied to their experts' rows
combine          the experts' rows added up per token with the router's weights
experts_back     the gradients of combine (rows and weights) and of dispatch
"""
import math

import numpy as np
import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)  # the quintic's coefficients
STEPS = 5
NORM_EPS = 1e-7
LN_EPS = 1e-5
MU, LR, DECAY = 0.95, 0.02, 0.01
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one small square matrix (a head's projection): fifteen dependent products, latency alone
        dict(name="orth_256x256_bf16", op="orthogonalize", dtype="bf16", batch=1, rows=256, cols=256),
        # the stacked matrices of a layer of 16 experts
        dict(name="orth_16x512x1408_bf16", op="orthogonalize", dtype="bf16", batch=16, rows=512, cols=1408),
        # a wide model's square projection
        dict(name="orth_4096x4096_bf16", op="orthogonalize", dtype="bf16", batch=1, rows=4096, cols=4096),
        # a server's iteration on an odd, tall matrix with fp32 gradient rows
        dict(name="step_1000x777_f32", op="step", dtype="f32", batch=1, rows=1000, cols=777, N=10, b=2),
        # a feed-forward matrix with bf16 gradient rows
        dict(name="step_2048x4096_bf16", op="step", dtype="bf16", batch=1, rows=2048, cols=4096, N=16, b=4),
        # a few tokens, odd width
        dict(name="ln_3x1023_f32", op="layer_norm", dtype="f32", tokens=3, width=1023),
        # a training batch's tokens
        dict(name="ln_8192x4096_bf16", op="layer_norm", dtype="bf16", tokens=8192, width=4096),
        # ragged batch, odd width, fp32
        dict(name="ln_back_777x1000_f32", op="layer_norm_back", dtype="f32", tokens=777, width=1000),
        dict(name="ln_back_8192x4096_bf16", op="layer_norm_back", dtype="bf16", tokens=8192, width=4096),
        # many small experts, eight to a token
        dict(name="dispatch_8192x2048_k8_bf16", op="dispatch", dtype="bf16", tokens=8192, width=2048, k=8, experts=64),
        # a small ragged batch, fp32, two experts to a token
        dict(name="combine_333x1000_k2_f32", op="combine", dtype="f32", tokens=333, width=1000, k=2, experts=8),
        dict(name="experts_back_8192x2048_k2_bf16", op="experts_back", dtype="bf16", tokens=8192, width=2048, k=2, experts=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _round_some(rng, n, to):
    """Half of the drawn sizes are multiples of `to`, the others what they are."""
    return max(to, n // to * to) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["orthogonalize", "step", "layer_norm", "layer_norm_back", "dispatch", "combine", "experts_back"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "orthogonalize":
        rows, cols = (_round_some(rng, _log(rng, 48, 4096), 64) for _ in range(2))
        most = max(1, min(32, int(4096 ** 3 * 0.5 / (min(rows, cols) ** 2 * max(rows, cols)))))
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, most), rows=rows, cols=cols)
    if op == "step":
        rows, cols = (_round_some(rng, _log(rng, 768, 2900), 64) for _ in range(2))
        return dict(op=op, dtype=dtype, batch=1, rows=rows, cols=cols, N=rng.randint(4, 16), b=rng.randint(0, 4))
    if op in ("layer_norm", "layer_norm_back"):
        width = _round_some(rng, _log(rng, 64, 8192), 64)
        return dict(op=op, dtype=dtype, tokens=_log(rng, 1, min(16384, 8192 * 2048 // width)), width=width)
    k = rng.randint(1, 8)
    width = _round_some(rng, _log(rng, 64, 8192), 64)
    tokens = _log(rng, 1, min(16384, 8192 * 4096 // (width * k)))
    return dict(op=op, dtype=dtype, tokens=tokens, width=width, k=k, experts=max(k, _log(rng, 4, 256)))


# ------------------------------------------------------------------ inputs


def _matrices(gen, batch, rows, cols):
    """A momentum's spectrum: noise with a few directions that stand out."""
    dev = "cuda"
    rank = min(8, rows, cols)
    u = torch.randn(batch, rows, cols, device=dev, generator=gen)
    left = torch.randn(batch, rows, rank, device=dev, generator=gen)
    right = torch.randn(batch, rank, cols, device=dev, generator=gen)
    return (u + 0.25 * left @ right) * 1e-3


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    host = np.random.Generator(np.random.Philox(seed))
    dt, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case)
    if op == "orthogonalize":
        s["u"] = _matrices(gen, case["batch"], case["rows"], case["cols"]).to(dt)
        s["out"] = torch.empty(s["u"].shape, dtype=torch.bfloat16, device=dev)
    elif op == "step":
        N, W = case["N"], case["N"] + case["b"]
        P = case["batch"] * case["rows"] * case["cols"]
        ld = (P + 7) // 8 * 8
        base = _matrices(gen, case["batch"], case["rows"], case["cols"]).reshape(P)
        s["grad"] = torch.empty(W, ld, dtype=dt, device=dev)
        for w in range(W):  # each worker's mini-batch: the common gradient and noise of its own
            s["grad"][w, :P] = base + 1e-3 * torch.randn(P, device=dev, generator=gen)
        s["arrival"] = torch.from_numpy(host.lognormal(0.0, 0.3, W).astype(np.float32)).to(dev)
        s["tags"] = torch.full((W,), 7, dtype=torch.int32, device=dev)
        s["theta"] = torch.randn(P, device=dev, generator=gen)
        s["momentum"] = 5.0 * base + 1e-3 * torch.randn(P, device=dev, generator=gen)
        s["mask"] = torch.empty(W, dtype=torch.uint8, device=dev)
        s["order"] = torch.empty(N, dtype=torch.int32, device=dev)
        s["info"] = torch.empty(2, dtype=torch.int32, device=dev)
    elif op in ("layer_norm", "layer_norm_back"):
        T, D = case["tokens"], case["width"]
        s["x"] = (torch.randn(T, D, device=dev, generator=gen) + 0.5 * torch.randn(D, device=dev, generator=gen)).to(dt)
        s["gamma"] = 1.0 + 0.1 * torch.randn(D, device=dev, generator=gen)
        s["beta"] = 0.1 * torch.randn(D, device=dev, generator=gen)
        if op == "layer_norm":
            s["y"] = torch.empty(T, D, dtype=dt, device=dev)
            s["mean"], s["rstd"] = torch.empty(T, device=dev), torch.empty(T, device=dev)
        else:
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = ((x - s["mean"][:, None]).square().mean(1) + LN_EPS).rsqrt()
            s["dy"] = (0.1 * torch.randn(T, D, device=dev, generator=gen)).to(dt)
            s["dx"] = torch.empty(T, D, dtype=dt, device=dev)
            s["dgamma"], s["dbeta"] = torch.empty(D, device=dev), torch.empty(D, device=dev)
    else:
        T, D, k, E = case["tokens"], case["width"], case["k"], case["experts"]
        # a router's choice: popular and unpopular experts, k different ones to a token, one pair in fifty over capacity
        logits = torch.randn(T, E, device=dev, generator=gen) + 0.7 * torch.randn(E, device=dev, generator=gen)
        top = torch.topk(logits, k, dim=1)
        ids = top.indices.to(torch.int32)
        ids[torch.rand(T, k, device=dev, generator=gen) < 0.02] = -1
        s["ids"], s["weights"] = ids.contiguous(), torch.softmax(top.values, 1).contiguous()
        s["offsets"] = torch.empty(E + 1, dtype=torch.int32, device=dev)
        s["slot"] = torch.empty(T, k, dtype=torch.int32, device=dev)
        s["source"] = torch.empty(T * k, dtype=torch.int32, device=dev)
        if op == "dispatch":
            s["x"] = torch.randn(T, D, device=dev, generator=gen).to(dt)
            s["xs"] = torch.empty(T * k, D, dtype=dt, device=dev)
        else:  # the router's plan is in hand by then
            offsets, slot, source = _plain_route(ids, E)
            s["offsets"].copy_(offsets)
            s["slot"].copy_(slot)
            s["source"].copy_(source)
            used = torch.arange(T * k, device=dev)[:, None] < offsets[-1]
            s["ys"] = (torch.randn(T * k, D, device=dev, generator=gen) * used).to(dt)
            s["out"] = torch.empty(T, D, dtype=dt, device=dev)
            if op == "experts_back":
                s["dout"] = (0.1 * torch.randn(T, D, device=dev, generator=gen)).to(dt)
                s["dxs"] = (0.1 * torch.randn(T * k, D, device=dev, generator=gen) * used).to(dt)
                s["dys"] = torch.empty(T * k, D, dtype=dt, device=dev)
                s["dweights"] = torch.empty(T, k, device=dev)
    return s


# ------------------------------------------------------------------ plain forms


def _plain_orthogonalize(u):
    a, b, c = COEF
    x = u / ((u * u).sum((-2, -1), keepdim=True).sqrt() + NORM_EPS)
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-2, -1) if tall else x
    for _ in range(STEPS):
        g = x @ x.transpose(-2, -1)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.transpose(-2, -1) if tall else x


def _plain_route(ids, E):
    """offsets [E+1], the row of each pair (-1: dropped), the pair of each row (-1: unused)."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    source = torch.argsort(key, stable=True)
    counts = (key[:, None] == torch.arange(E, device=ids.device)).sum(0) if key.numel() * E < 1 << 24 else torch.bincount(key, minlength=E + 1)[:E]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    place = torch.empty_like(source)
    place[source] = torch.arange(source.numel(), device=ids.device)
    slot = torch.where(key < E, place, -1)
    source = torch.where(torch.arange(source.numel(), device=ids.device) < offsets[-1], source, -1)
    return offsets.int(), slot.reshape(ids.shape).int(), source.int()


def _plain_gather(rows, slot):
    """rows [S, D], slot [T, k] -> fp32 [T, k, D], zero where the pair was dropped."""
    return rows.float()[slot.long().clamp(min=0)] * (slot >= 0)[..., None]


def _plain(s):
    op, dt = s["op"], DTYPES[s["dtype"]]
    if op == "orthogonalize":
        return [_plain_orthogonalize(s["u"].float()).to(torch.bfloat16)]
    if op == "step":
        P = s["theta"].numel()
        # the first N to arrive among those tagged with this iteration (all are, here)
        order = torch.argsort(s["arrival"], stable=True)[: s["N"]]
        g = s["grad"][order, :P].float().sum(0) / s["N"]
        s["momentum"].mul_(MU).add_(g)
        u = (g + MU * s["momentum"]).view(s["batch"], s["rows"], s["cols"])
        o = _plain_orthogonalize(u).reshape(P)
        scale = math.sqrt(max(1.0, s["rows"] / s["cols"]))
        s["theta"].mul_(1.0 - LR * DECAY).sub_(LR * scale * o)
        return [s["theta"], s["momentum"]]
    if op == "layer_norm":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = (d.square().mean(1) + LN_EPS).rsqrt()
        return [(d * rstd[:, None] * s["gamma"] + s["beta"]).to(dt), mean, rstd]
    if op == "layer_norm_back":
        dy = s["dy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        h = dy * s["gamma"]
        dx = s["rstd"][:, None] * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
        return [dx.to(dt), (dy * xh).sum(0), dy.sum(0)]
    if op == "dispatch":
        offsets, slot, source = _plain_route(s["ids"], s["experts"])
        xs = s["x"].float()[(source.long().clamp(min=0)) // s["k"]] * (source >= 0)[:, None]
        return [offsets, slot, source, xs.to(dt)]
    if op == "combine":
        return [(_plain_gather(s["ys"], s["slot"]) * s["weights"][..., None]).sum(1).to(dt)]
    source, used = s["source"].long().clamp(min=0), s["source"] >= 0
    dout = s["dout"].float()
    dys = dout[source // s["k"]] * (s["weights"].reshape(-1)[source] * used)[:, None]
    dweights = (_plain_gather(s["ys"], s["slot"]) * dout[:, None, :]).sum(2)
    dx = _plain_gather(s["dxs"], s["slot"]).sum(1)
    return [dys.to(dt), dweights, dx.to(dt)]


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    from paper_1604_00981_b200 import binding as sgdb

    op = s["op"]
    if op in ("orthogonalize", "step", "layer_norm_back") and "workspace" not in s:  # kept from pass to pass, as a training loop does
        if op == "layer_norm_back":
            need = sgdb.sgdb_layer_norm_backward_workspace_bytes(s["tokens"], s["width"])
        else:
            of = sgdb.sgdb_orthogonalize_workspace_bytes if op == "orthogonalize" else sgdb.sgdb_step_orthogonal_workspace_bytes
            need = of(s["batch"], s["rows"], s["cols"])
        s["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    if op == "orthogonalize":
        sgdb.sgdb_orthogonalize(s["u"], s["out"], sgdb.NewtonSchulz(STEPS, *COEF, NORM_EPS), s["workspace"])
        return [s["out"]]
    if op == "step":
        opt = sgdb.OrthogonalOpt(lr=LR, momentum=MU, nesterov=True, weight_decay=DECAY, scale=math.sqrt(max(1.0, s["rows"] / s["cols"])),
                                 newton_schulz=sgdb.NewtonSchulz(STEPS, *COEF, NORM_EPS))
        sgdb.sgdb_step_orthogonal(s["grad"], s["batch"], s["rows"], s["cols"], s["arrival"], s["tags"], 7, s["N"], s["b"], s["theta"],
                                  s["momentum"], opt, s["mask"], s["order"], s["info"], s["workspace"])
        return [s["theta"], s["momentum"]]
    if op == "layer_norm":
        sgdb.sgdb_layer_norm(s["x"], s["gamma"], s["beta"], LN_EPS, s["y"], s["mean"], s["rstd"])
        return [s["y"], s["mean"], s["rstd"]]
    if op == "layer_norm_back":
        sgdb.sgdb_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["workspace"])
        return [s["dx"], s["dgamma"], s["dbeta"]]
    if op == "dispatch":
        sgdb.sgdb_route(s["ids"], s["experts"], s["offsets"], s["slot"], s["source"])
        sgdb.sgdb_dispatch(s["x"], s["slot"], s["offsets"], s["xs"])
        return [s["offsets"], s["slot"], s["source"], s["xs"]]
    if op == "combine":
        sgdb.sgdb_combine(s["ys"], s["slot"], s["weights"], s["out"])
        return [s["out"]]
    sgdb.sgdb_combine_backward(s["dout"], s["ys"], s["slot"], s["weights"], s["offsets"], s["dys"], s["dweights"])
    sgdb.sgdb_combine(s["dxs"], s["slot"], None, s["out"])  # the gradient of dispatch
    return [s["dys"], s["dweights"], s["out"]]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op in ("orthogonalize", "step"):
        m, n = sorted((case["rows"], case["cols"]))
        P = case["batch"] * m * n
        # the Gram matrix and its square are symmetric: half of their products
        flops = case["batch"] * STEPS * (m * m * n + m * m * m + 2 * m * m * n)
        if op == "orthogonalize":
            return {"bytes": P * (size + 2), "flops": flops}
        return {"bytes": P * (case["N"] * size + 16), "flops": flops + P * case["N"]}
    T, D = case["tokens"], case["width"]
    if op == "layer_norm":
        return {"bytes": 2 * T * D * size + 8 * D + 8 * T, "flops": 8 * T * D}
    if op == "layer_norm_back":
        return {"bytes": 3 * T * D * size + 12 * D + 8 * T, "flops": 15 * T * D}
    k, E = case["k"], case["experts"]
    rows = T * k * D * size
    if op == "dispatch":
        return {"bytes": T * D * size + rows + 12 * T * k + 4 * E, "flops": T * k}
    if op == "combine":
        return {"bytes": T * D * size + rows + 8 * T * k, "flops": 2 * T * k * D}
    return {"bytes": 2 * T * D * size + 3 * rows + 12 * T * k, "flops": 4 * T * k * D}


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_orthogonal(u):
    """p(p(..p(U/|U|))) with p(X) = X (aI + bG + cG^2), G = X^T X over the shorter side."""
    a, b, c = COEF
    flip = u.shape[-1] > u.shape[-2]
    z = u.double()
    z = z.mT if flip else z
    z = z / (torch.linalg.matrix_norm(z, keepdim=True) + NORM_EPS)
    eye = torch.eye(z.shape[-1], dtype=torch.float64, device=z.device)
    for _ in range(STEPS):
        gram = z.mT @ z
        z = z @ (a * eye + gram @ (b * eye + c * gram))
    return z.mT if flip else z


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "orthogonalize":
        return [_exact_orthogonal(s["u"])]
    if op == "step":
        P, N = s["theta"].numel(), case["N"]
        kept = sorted(range(len(s["arrival"])), key=lambda w: (float(s["arrival"][w]), w))[:N]
        mean = torch.zeros(P, dtype=torch.float64, device="cuda")
        for w in kept:
            mean += s["grad"][w, :P].double() / N
        velocity = MU * s["momentum"].double() + mean
        o = _exact_orthogonal((mean + MU * velocity).view(case["batch"], case["rows"], case["cols"])).reshape(P)
        return [s["theta"].double() * (1 - LR * DECAY) - LR * math.sqrt(max(1.0, case["rows"] / case["cols"])) * o, velocity]
    if op == "layer_norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + LN_EPS)
        return [torch.addcmul(s["beta"].double(), (x - mean[:, None]) * rstd[:, None], s["gamma"].double()), mean, rstd]
    if op == "layer_norm_back":
        # the Jacobian applied with the statistics as they were handed over
        r, D = s["rstd"].double(), case["width"]
        n = (s["x"].double() - s["mean"].double()[:, None]) * r[:, None]
        dy = s["dy"].double()
        h = torch.einsum("td,d->td", dy, s["gamma"].double())
        along = torch.einsum("td,td->t", h, n) / D
        return [(h - (h.sum(1) / D)[:, None] - n * along[:, None]) * r[:, None], torch.einsum("td,td->d", dy, n), dy.sum(0)]
    T, D, k, E = case["tokens"], case["width"], case["k"], case["experts"]
    ids = s["ids"].reshape(-1).cpu().numpy()
    fits = (ids >= 0) & (ids < E)
    rows = np.lexsort((np.arange(T * k), np.where(fits, ids, E)))[: int(fits.sum())]  # pairs in the experts' order
    source = torch.from_numpy(rows).cuda()
    if op == "dispatch":
        slot = np.full(T * k, -1, np.int32)
        slot[rows] = np.arange(rows.size)
        back = np.full(T * k, -1, np.int32)
        back[: rows.size] = rows
        offsets = np.searchsorted(ids[rows], np.arange(E + 1)).astype(np.int32)
        xs = torch.zeros(T * k, D, dtype=torch.float64, device="cuda")
        xs[: rows.size] = s["x"].double()[source // k]
        return [offsets, slot.reshape(T, k), back, xs]
    w = s["weights"].double().reshape(-1)[source]
    ys = s["ys"].double()[: rows.size]
    if op == "combine":
        return [torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, source // k, ys * w[:, None])]
    dout = s["dout"].double()[source // k]
    dys = torch.zeros(T * k, D, dtype=torch.float64, device="cuda")
    dys[: rows.size] = dout * w[:, None]
    dweights = torch.zeros(T * k, dtype=torch.float64, device="cuda")
    dweights[source] = (dout * ys).sum(1)
    dx = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, source // k, s["dxs"].double()[: rows.size])
    return [dys, dweights.reshape(T, k), dx]
