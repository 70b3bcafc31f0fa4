"""The layer of experts in 8 bits through autograd, with all its operators together, under graphs, on other streams and devices.

The reference computes the same layer in 64 bits with the same roundings to 8 bits, which the backward pass takes as the identity.
In fp32 both see the same numbers up to 1e-6, and a number next to a border between two 8-bit numbers goes to the other side for about one
in 1e5 (a step of 2^-4 over 1e-6): the norm of the difference is below sqrt(1e-5) 2^-4 = 2e-4 of the result's per rounding, three roundings deep."""
import contextlib
import importlib.util
import os

import pytest
import torch

import f8_helpers as f8
from paper_1604_00981_b200 import binding as sgdb
from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu


class Round(torch.autograd.Function):
    """To 8 bits along the last dimension; the gradient goes through, rounded too where it is an operand."""
    @staticmethod
    def forward(ctx, x, fmt):
        q, e = f8.quantized(x.float(), fmt)
        return f8.wide(q, torch.exp2(e))

    @staticmethod
    def backward(ctx, g):
        return g, None


def rounded(x, fmt):
    return Round.apply(x, fmt)


class RoundMatrices(torch.autograd.Function):
    @staticmethod
    def forward(ctx, w, fmt):
        q, e = f8.quantized_matrices(w.float(), fmt)
        return f8.wide_matrices(q, torch.exp2(e))

    @staticmethod
    def backward(ctx, g):
        return g, None


class Product(torch.autograd.Function):
    """x W^T with both gradients as the layer takes them: of the rows from dy in 8 bits, of the matrices from dy as it is."""
    @staticmethod
    def forward(ctx, x, w, fmt):
        ctx.save_for_backward(x, w)
        ctx.fmt = fmt
        return x @ w.T

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        return rounded(dy, ctx.fmt) @ w, dy.T @ x, None


class Gate(torch.autograd.Function):
    """silu(g) u whose gradient is taken at h in 8 bits."""
    @staticmethod
    def forward(ctx, h, fmt):
        q, e = f8.quantized(h.float().unflatten(1, (2, h.size(1) // 2)), fmt)
        ctx.save_for_backward(f8.wide(q, torch.exp2(e)))
        g, u = h.chunk(2, 1)
        return g / (1 + torch.exp(-g)) * u

    @staticmethod
    def backward(ctx, da):
        (h,) = ctx.saved_tensors
        g, u = h[:, 0], h[:, 1]
        sig = 1 / (1 + torch.exp(-g))
        return torch.cat([da * u * sig * (1 + g * (1 - sig)), da * g * sig], 1), None


def reference(xs, up, down, edges, fmt):
    out = []
    for e, (a, b) in enumerate(zip(edges, edges[1:])):
        h = Product.apply(rounded(xs[a:b], fmt), RoundMatrices.apply(up[e][None], fmt)[0], fmt)
        out.append(Product.apply(rounded(Gate.apply(h, fmt), fmt), RoundMatrices.apply(down[e][None], fmt)[0], fmt))
    return torch.cat(out + [torch.zeros_like(xs[edges[-1]:])])


def inputs(T, D, F, E, k, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    ids = torch.randint(-1, E, (T, k), device="cuda", generator=gen).int()
    return new(T, D), new(E, 2 * F, D) * D ** -0.5, new(E, D, F) * F ** -0.5, new(T, k), ids


def distance(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("fmt", f8.FORMATS)
@pytest.mark.parametrize("T,D,F,E,k", [(60, 96, 80, 5, 2), (1, 64, 48, 8, 8), (700, 256, 384, 3, 2), (37, 200, 136, 40, 1)])
def test_against_64_bits(cuda_device, T, D, F, E, k, fmt):
    x, up, down, weights, ids = inputs(T, D, F, E, k)
    r = layers.route(ids, E)
    edges = r.offsets.tolist()

    def leaves(dtype):
        return [v.to(dtype).detach().requires_grad_() for v in (x, up, down, weights)]

    a = leaves(torch.float32)
    ys = layers.experts(layers.dispatch(a[0], r), a[1], a[2], r, fmt)
    out = layers.combine(ys, a[3], r)
    (out * x.flip(0)).sum().backward()
    c = leaves(torch.float64)
    source = r.source[: edges[-1]].long()
    xs = torch.cat([c[0][source // k], torch.zeros(T * k - edges[-1], D, dtype=torch.float64, device="cuda")])
    ys = reference(xs, c[1], c[2], edges, fmt)
    ref = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add(0, source // k, ys[: edges[-1]] * c[3].reshape(-1)[source, None])
    (ref * x.flip(0).double()).sum().backward()
    assert distance(out.detach(), ref.detach()) <= 1e-3
    for got, want in zip(a, c):
        assert got.grad.dtype == torch.float32 and distance(got.grad, want.grad) <= 2e-3


def test_bf16_and_which_gradients(cuda_device):
    """bf16 rows with fp32 matrices; each input alone; an experts' output of rows not in use is zero."""
    x, up, down, weights, ids = inputs(90, 128, 160, 4, 2)
    r = layers.route(ids, 4)
    xs = layers.dispatch(x.bfloat16(), r)
    whole = [xs.detach().requires_grad_(), up.requires_grad_(), down.requires_grad_()]
    ys = layers.experts(*whole, r)
    used = int(r.offsets[-1])
    assert ys.dtype == torch.bfloat16 and used < 180 and not bool(ys[used:].any())
    g = torch.randn_like(ys)
    want = torch.autograd.grad(ys, whole, g)
    assert [w.dtype for w in want] == [torch.bfloat16, torch.float32, torch.float32] and not bool(want[0][used:].any())
    for i in range(3):
        alone = [v.detach().requires_grad_(j == i) for j, v in enumerate(whole)]
        ys = layers.experts(*alone, r)
        (got,) = torch.autograd.grad(ys, alone[i], g)
        assert torch.equal(got, want[i])
    with pytest.raises(ValueError):
        layers.experts(xs, up[:, :-1], down, r)
    with pytest.raises(RuntimeError):
        (d,) = torch.autograd.grad(layers.experts(*whole, r), whole[0], g, create_graph=True)
        d.sum().backward()


def test_any_strides(cuda_device):
    x, up, down, _, ids = inputs(50, 96, 64, 3, 2)
    r = layers.route(ids, 3)
    xs = layers.dispatch(x, r)
    want = layers.experts(xs, up, down, r)
    g = torch.randn_like(want)
    odd = [torch.empty(100, 99, device="cuda")[:, 3:].copy_(xs).requires_grad_(), up.mT.contiguous().mT.requires_grad_(), down.mT.contiguous().mT.requires_grad_()]
    got = layers.experts(*odd, r)
    assert torch.equal(got, want)
    plain = [xs.detach().requires_grad_(), up.requires_grad_(), down.requires_grad_()]
    a = torch.autograd.grad(got, odd, g.t().contiguous().t())
    b = torch.autograd.grad(layers.experts(*plain, r), plain, g)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_no_tokens_and_nobody_chosen(cuda_device):
    """No rows at all, and rows that all belong to nobody: zeros, and gradients of zeros."""
    x, up, down, weights, ids = inputs(8, 64, 48, 3, 2)
    for T in (0, 8):
        leaves = [v.detach().requires_grad_() for v in (x[:T], up, down)]
        r = layers.route(torch.full((T, 2), -1, dtype=torch.int32, device="cuda"), 3)
        ys = layers.experts(layers.dispatch(leaves[0], r), leaves[1], leaves[2], r)
        assert ys.shape == (2 * T, 64) and not bool(ys.any())
        for g, v in zip(torch.autograd.grad(ys, leaves, torch.ones_like(ys)), leaves):
            assert g.shape == v.shape and not bool(g.any())
    loss, counts = layers.balance_loss(x[:0, :3], ids[:0])
    assert float(loss) == 0.0 and counts.tolist() == [0, 0, 0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_balance_loss_layer(cuda_device, dtype):
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn(70, 6, device="cuda", generator=gen).to(dtype)
    ids = torch.topk(logits, 2, dim=1).indices.int()
    mask = torch.rand(70, device="cuda", generator=gen) < 0.8
    for m in (None, mask):
        for x in (logits, logits.t().contiguous().t(), torch.empty(70, 9, device="cuda", dtype=dtype)[:, 2:8].copy_(logits)):
            x = x.detach().requires_grad_()
            loss, counts = layers.balance_loss(x, ids, m)
            (3.0 * loss).backward()
            c = logits.double().requires_grad_()
            kept = torch.ones_like(mask) if m is None else m
            n = int(kept.sum())
            count = torch.bincount(ids[kept].reshape(-1).long(), minlength=6)
            want = 6 * ((count.double() / (2 * n)) * torch.softmax(c, 1)[kept].mean(0)).sum()
            (3.0 * want).backward()
            assert torch.equal(counts.long(), count) and abs(float(loss.detach() - want.detach())) <= 1e-5 * float(want.detach())
            # probabilities and bracket within 2^-17 of the largest gradient, one rounding to the type
            bound = 2.0 ** -17 * float(c.grad.abs().max()) + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * c.grad.abs()
            assert bool(((x.grad.double() - c.grad).abs() <= bound).all())


def everything(T, D, F, E, k, dtype, fmt):
    """One worker's forward and backward pass with all the operators, by the binding's calls on arrays that stay where they are."""
    new = lambda *s: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    e8 = lambda *s: sgdb.empty_f8(*s, dtype=fmt, device="cuda")  # noqa: E731
    sc = lambda *s: sgdb.empty_scale(*s, device="cuda")  # noqa: E731
    mat = lambda R, C: torch.empty(E, (R + 127) // 128, (C + 127) // 128, dtype=torch.float8_e8m0fnu, device="cuda")  # noqa: E731
    S = T * k
    a = dict(x=new(T, D), up=f32(E, 2 * F, D), down=f32(E, D, F), w=f32(T, k), dout=new(T, D), logits=new(T, E))
    ids, grad = i32(T, k), torch.full((1,), 0.01, device="cuda")
    o = dict(loss=f32(1), counts=i32(E), slope=f32(E), dlogits=new(T, E), offsets=i32(E + 1), slot=i32(T, k), source=i32(S), xs=new(S, D), h=new(S, 2 * F),
             ys=new(S, D), out=new(T, D), dys=new(S, D), dw=f32(T, k), da=new(S, F), dh=new(S, 2 * F), dxs=new(S, D), dx=new(T, D), dup=f32(E, 2 * F, D),
             ddown=new(E, D, F))
    x8, xs8, up8, up8t, ups, down8, down8t, downs = e8(S, D), sc(S, D), e8(E, 2 * F, D), e8(E, D, 2 * F), mat(2 * F, D), e8(E, D, F), e8(E, F, D), mat(D, F)
    a8, as8, h8, hs8, dy8, dys8, dh8, dhs8 = e8(S, F), sc(S, F), e8(S, 2, F), sc(S, 2, F), e8(S, D), sc(S, D), e8(S, 2 * F), sc(S, 2 * F)
    byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    ws = byte(max(sgdb.sgdb_balance_loss_workspace_bytes(T, E), sgdb.sgdb_experts_gradient_workspace_bytes(S, 2 * F, D, E),
                  sgdb.sgdb_experts_gradient_workspace_bytes(S, D, F, E)))

    def call():
        sgdb.sgdb_balance_loss(a["logits"], ids, None, o["loss"], o["counts"], o["slope"], ws)
        sgdb.sgdb_route(ids, E, o["offsets"], o["slot"], o["source"])
        sgdb.sgdb_dispatch(a["x"], o["slot"], o["offsets"], o["xs"])
        sgdb.sgdb_quantize_matrices(a["up"], up8, up8t, ups)
        sgdb.sgdb_quantize_matrices(a["down"], down8, down8t, downs)
        sgdb.sgdb_quantize(o["xs"], x8, xs8)
        sgdb.sgdb_experts_product(x8, xs8, up8, ups, o["offsets"], o["h"])
        sgdb.sgdb_gate(o["h"], a8, as8, h8, hs8)
        sgdb.sgdb_experts_product(a8, as8, down8, downs, o["offsets"], o["ys"])
        sgdb.sgdb_combine(o["ys"], o["slot"], a["w"], o["out"])
        sgdb.sgdb_combine_backward(a["dout"], o["ys"], o["slot"], a["w"], o["offsets"], o["dys"], o["dw"])
        sgdb.sgdb_quantize(o["dys"], dy8, dys8)
        sgdb.sgdb_experts_product(dy8, dys8, down8t, downs.transpose(1, 2), o["offsets"], o["da"])
        sgdb.sgdb_experts_gradient(o["dys"], a8, as8, o["offsets"], o["ddown"], ws)
        sgdb.sgdb_gate_backward(o["da"], h8, hs8, o["dh"])
        sgdb.sgdb_quantize(o["dh"], dh8, dhs8)
        sgdb.sgdb_experts_product(dh8, dhs8, up8t, ups.transpose(1, 2), o["offsets"], o["dxs"])
        sgdb.sgdb_experts_gradient(o["dh"], x8, xs8, o["offsets"], o["dup"], ws)
        sgdb.sgdb_combine(o["dxs"], o["slot"], None, o["dx"])
        sgdb.sgdb_balance_loss_backward(grad, a["logits"], None, o["slope"], o["dlogits"])

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for v in a.values():
            v.copy_(torch.randn(v.shape, device="cuda", generator=gen))
        ids.copy_(torch.randint(-1, E + 1, (T, k), device="cuda", generator=gen))

    return call, fill, list(o.values())


SHAPES = {"ragged": (75, 72, 56, 5, 2, torch.float32, torch.float8_e5m2), "many rows": (4096, 256, 136, 2, 2, torch.bfloat16, torch.float8_e4m3fn),
          "one token": (1, 1024, 512, 64, 8, torch.bfloat16, torch.float8_e4m3fn)}


@pytest.mark.parametrize("case", SHAPES)
def test_replays(cuda_device, case):
    """All of them captured in a graph, twice, with one workspace: replays in turn, with other inputs in the same arrays, give the plain calls' bits."""
    call, fill, outputs = everything(*SHAPES[case])
    want = {}
    for seed in (1, 2, 3):
        fill(seed)
        call()
        want[seed] = [v.clone() for v in outputs]
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        fill(1)
        torch.cuda.synchronize()
        with torch.cuda.graph(graphs[-1]):
            call()
    for i, seed in enumerate((2, 3, 2, 1, 3)):
        fill(seed)
        for v in outputs:
            v.fill_(1)
        graphs[i % 2].replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want[seed]))


def test_another_stream(cuda_device):
    call, fill, outputs = everything(*SHAPES["ragged"])
    fill(1)
    call()
    want = [v.clone() for v in outputs]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        fill(2)
        fill(1)
        call()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))


def test_a_captured_training_step(cuda_device):
    """The layers' forward and backward pass under capture, with leaves of its own: torch does not capture a backward pass whose
    leaves belong to an eager graph that still lives."""
    x, up, down, weights, ids = inputs(64, 96, 64, 4, 2)
    r = layers.route(ids, 4)

    def step(leaves):
        out = layers.combine(layers.experts(layers.dispatch(leaves[0], r), leaves[1], leaves[2], r), leaves[3], r)
        return torch.autograd.grad((out * out).sum(), leaves)

    fresh = lambda: [v.detach().requires_grad_() for v in (x, up, down, weights)]  # noqa: E731
    want = step(fresh())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(fresh())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(fresh())
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_tensors_of_another_device(cuda_device, monkeypatch):
    S, D, E = 6, 32, 2
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    e8, sc = lambda *s: sgdb.empty_f8(*s, device="cuda").fill_(0), lambda *s: sgdb.empty_scale(*s, device="cuda").fill_(1.0)  # noqa: E731
    off = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    ms = torch.ones(E, 1, 1, device="cuda").to(torch.float8_e8m0fnu)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    ids, i32 = torch.zeros(S, 1, dtype=torch.int32, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")
    calls = [lambda: sgdb.sgdb_quantize(f(S, D), e8(S, D), sc(S, D)), lambda: sgdb.sgdb_quantize_matrices(f(E, D, D), e8(E, D, D), None, ms),
             lambda: sgdb.sgdb_gate(f(S, 2 * D), e8(S, D), sc(S, D), e8(S, 2, D), sc(S, 2, D)),
             lambda: sgdb.sgdb_gate_backward(f(S, D), e8(S, 2, D), sc(S, 2, D), f(S, 2 * D)),
             lambda: sgdb.sgdb_experts_product(e8(S, D), sc(S, D), e8(E, D, D), ms, off, f(S, D)),
             lambda: sgdb.sgdb_experts_gradient(f(S, D), e8(S, D), sc(S, D), off, f(E, D, D), ws),
             lambda: sgdb.sgdb_balance_loss(f(S, E), ids, None, f(1), i32, f(E), ws), lambda: sgdb.sgdb_balance_loss_backward(f(1), f(S, E), None, f(E), f(S, E))]
    for call in calls:
        call()
    x, up, down, weights, idx = inputs(S, 64, 64, 2, 1)
    xs = x.requires_grad_()

    def layer():
        r = layers.route(idx, 2)
        return layers.experts(xs, up, down, r), layers.balance_loss(xs[:, :2], idx)[0]

    want = layer()
    entered = []

    @contextlib.contextmanager
    def device(d):
        entered.append(d)
        yield

    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        m.setattr(torch.cuda, "device", device)
        got = layer()
        assert len(entered) == 3 and all(torch.equal(a, b) for a, b in zip(got, want))
        torch.autograd.grad(got[0].sum() + got[1], xs)
        assert len(entered) == 5
    monkeypatch.setattr(sgdb, "_current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()


def test_the_training_example(cuda_device):
    """It runs with both kinds of gradient rows, and its block's gradients are those of the same block in 64 bits with the same roundings."""
    spec = importlib.util.spec_from_file_location("train_experts", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                                                                                "train_experts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for dtype in (torch.float32, torch.bfloat16):
        losses = example.train(steps=3, dtype=dtype, eight_bit=True)
        assert len(losses) == 3 and all(0.0 < v < 100.0 for v in losses)
    gen = torch.Generator(device="cuda").manual_seed(3)
    p = {n: torch.randn(s, device="cuda", generator=gen) * (0.3 if len(s) > 1 else 1.0) for n, s in example.shapes(True).items()}
    tokens = torch.randint(0, example.CLASSES, (example.TOKENS,), device="cuda", generator=gen)
    targets = tokens.flip(0)
    a = {n: v.clone().requires_grad_() for n, v in p.items()}
    example.forward(a, tokens, targets, True).backward()
    c = {n: v.double().requires_grad_() for n, v in p.items()}
    x = c["embed"][tokens]
    mean = x.mean(-1, keepdim=True)
    h = (x - mean) / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + 1e-5) * c["gamma"] + c["beta"]
    logits = h @ c["router"]
    top = torch.topk(logits, example.CHOICES, dim=1)
    E, k, T = example.EXPERTS, example.CHOICES, example.TOKENS
    order = torch.argsort(top.indices.reshape(-1), stable=True)
    counts = torch.bincount(top.indices.reshape(-1), minlength=E)
    edges = [0] + counts.cumsum(0).tolist()
    ys = reference(h[order // k], c["up"], c["down"], edges, torch.float8_e4m3fn)
    y = torch.zeros_like(x).index_add(0, order // k, ys * torch.softmax(top.values, 1).reshape(-1)[order, None])
    balance = E * ((counts.double() / (T * k)) * torch.softmax(logits, 1).mean(0)).sum()
    (torch.nn.functional.cross_entropy((x + y) @ c["out"], targets) + 0.01 * balance).backward()
    for n in p:
        assert distance(a[n].grad, c[n].grad) <= 2e-3, n
