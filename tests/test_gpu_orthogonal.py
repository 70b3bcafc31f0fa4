"""The orthogonalised update against the iteration in 64 bits, closed forms, and the framework's own elementwise calls.

Tolerances (Frobenius norm, relative): the products run on fp16 operands.  Rounding X, A and B to 11 bits in a simulation of
the iteration on the CPU leaves 1.2e-3 .. 2.1e-3 for random matrices whose shorter side is 32 or more and up to 1e-2 for
smaller ones, where the roundings do not average out; twice that is allowed.  Rounding the result to bf16 adds 1.7e-3."""
import math

import numpy as np
import pytest
import torch

from helpers import rel_err, selection_buffers
from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
NS = sgdb.NewtonSchulz()


def tolerance(side, dtype=torch.float32):
    t = 4e-3 if side >= 32 else 2e-2
    return math.hypot(t, 1.7e-3) if dtype == torch.bfloat16 else t


def reference(u, ns=NS):
    x = u.double()
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + ns.eps)
    for _ in range(ns.steps):
        if x.size(-2) <= x.size(-1):
            a = x @ x.mT
            x = ns.a * x + (ns.b * a + ns.c * a @ a) @ x
        else:
            a = x.mT @ x
            x = ns.a * x + x @ (ns.b * a + ns.c * a @ a)
    return x


def workspace(B, R, C, step=False):
    f = sgdb.sgdb_step_orthogonal_workspace_bytes if step else sgdb.sgdb_orthogonalize_workspace_bytes
    return torch.randint(0, 255, (f(B, R, C),), dtype=torch.uint8, device="cuda")  # what it holds does not matter


def off(x, y):
    return float((x.double() - y).norm() / y.norm())


SHAPES = [(1, 1, 1), (2, 1, 5), (2, 5, 1), (3, 7, 3), (1, 16, 40), (2, 33, 65), (1, 64, 64), (1, 65, 130), (2, 130, 65), (1, 128, 128), (2, 127, 129),
          (1, 129, 127), (5, 256, 256), (1, 256, 512), (1, 300, 1000), (1, 1000, 300), (1, 777, 1000), (2, 513, 520), (1, 64, 4096), (1, 4096, 72),
          (1, 1537, 1400), (40, 96, 200), (1, 31, 5000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,R,C", SHAPES)
def test_against_64_bits(cuda_device, B, R, C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(R * 31 + C)
    u = (torch.randn(B, R, C, device="cuda", generator=gen) * torch.logspace(-6, 6, B, device="cuda")[:, None, None]).to(dtype)
    ws = workspace(B, R, C)
    for dt_out in (torch.float32, torch.bfloat16):
        out = torch.full((B, R, C), 9.0, dtype=dt_out, device="cuda")
        sgdb.sgdb_orthogonalize(u, out, NS, ws)
        ref = reference(u)
        for b in range(B):
            assert off(out[b], ref[b]) <= tolerance(min(R, C), dt_out), (b, off(out[b], ref[b]))
        again = torch.empty_like(out)
        sgdb.sgdb_orthogonalize(u, again, NS, ws)
        assert torch.equal(out, again)


@pytest.mark.parametrize("R,C", [(40, 70), (70, 40), (128, 256), (257, 128)])
def test_strides_guards_and_in_place(cuda_device, R, C):
    B, pad, gap = 3, 5, 3
    whole = torch.full((B, R + gap, C + pad), 7.0, device="cuda")
    u = whole[:, :R, :C]
    u.copy_(torch.randn(B, R, C, device="cuda"))
    dense = u.contiguous()
    ref, ws = reference(dense), workspace(B, R, C)
    got = torch.empty_like(dense)
    sgdb.sgdb_orthogonalize(dense, got, NS, ws)
    out = torch.full((B, R + gap, C + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    sgdb.sgdb_orthogonalize(u, out[:, :R, :C], NS, ws)
    assert torch.equal(out[:, :R, :C], got.bfloat16())
    assert bool((out[:, R:] == 7.0).all()) and bool((out[:, :, C:] == 7.0).all())
    sgdb.sgdb_orthogonalize(u, u, NS, ws)
    assert torch.equal(u, got) and bool((whole[:, R:] == 7.0).all()) and bool((whole[:, :, C:] == 7.0).all())
    assert off(got, ref) <= tolerance(min(R, C))
    sgdb.sgdb_orthogonalize(dense[1], got[0], NS, ws)  # a single matrix
    assert torch.equal(got[0], got[1])


def test_orthogonal_matrix_goes_through_the_scalar_polynomial(cuda_device):
    """U = q P with P a permutation: every singular value is 1/sqrt(n) of |U|, so O = p(p(..p(1/sqrt(n)))) P."""
    n = 192
    u = torch.zeros(n, n, device="cuda")
    u[torch.arange(n), torch.randperm(n, generator=torch.Generator().manual_seed(1))] = -3.0
    v = 1 / math.sqrt(n)
    for _ in range(NS.steps):
        v = NS.a * v + NS.b * v ** 3 + NS.c * v ** 5
    out = torch.empty_like(u)
    sgdb.sgdb_orthogonalize(u, out, NS, workspace(1, n, n))
    # one diagonal value per matrix: its roundings do not average out over elements
    assert float((out - v * u / 3.0).abs().max()) <= 2e-2 * abs(v)
    assert bool((out[u == 0] == 0).all())


@pytest.mark.parametrize("steps,coef", [(1, (3.4445, -4.775, 2.0315)), (2, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))])
def test_other_polynomials(cuda_device, steps, coef):
    ns = sgdb.NewtonSchulz(steps, *coef)
    u = torch.randn(2, 96, 160, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    out = torch.empty_like(u)
    sgdb.sgdb_orthogonalize(u, out, ns, workspace(2, 96, 160))
    assert off(out, reference(u, ns)) <= 4e-3
    if steps == 12:  # the cubic converges: the rows are orthonormal
        assert float((out @ out.mT - torch.eye(96, device="cuda")).abs().max()) < 1e-2


def test_zero_and_non_finite_matrices_stay_by_themselves(cuda_device):
    B, R, C = 5, 72, 136
    u = torch.randn(B, R, C, device="cuda")
    clean = torch.empty_like(u)
    ws = workspace(B, R, C)
    sgdb.sgdb_orthogonalize(u, clean, NS, ws)
    u[0] = 0
    u[2, 3, 4] = float("nan")
    u[3, 71, 135] = float("-inf")
    out = torch.empty_like(u)
    sgdb.sgdb_orthogonalize(u, out, NS, ws)
    assert bool((out[0] == 0).all())
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3]).all())
    assert torch.equal(out[1], clean[1]) and torch.equal(out[4], clean[4])
    # squares outside fp32's range
    for scale in (1e-30, 1e30):
        big = u[1:2] * scale
        sgdb.sgdb_orthogonalize(big, out[1:2], sgdb.NewtonSchulz(eps=0.0), ws)
        assert off(out[1], reference(u[1], sgdb.NewtonSchulz(eps=0.0))) <= tolerance(72)


def test_info_word(cuda_device):
    u = torch.randn(48, 64, device="cuda")
    out = torch.full_like(u, 5.0)
    ws = workspace(1, 48, 64)
    info = torch.tensor([0, sgdb.SGDB_ERR_INSUFFICIENT], dtype=torch.int32, device="cuda")
    sgdb.sgdb_orthogonalize(u, out, NS, ws, info)
    assert bool((out == 5.0).all())
    info.zero_()
    sgdb.sgdb_orthogonalize(u, out, NS, ws, info)
    assert info.cpu().tolist() == [0, 0] and off(out, reference(u)) <= tolerance(48)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("B,R,C", [(1, 100, 77), (3, 64, 130), (1, 600, 256)])
def test_step(cuda_device, B, R, C, nesterov, dtype):
    N, b, P = 5, 2, B * R * C
    W, ld, dev = N + b, P + 13 if dtype == torch.float32 else (P + 7) // 8 * 8, "cuda"
    gen = torch.Generator(device=dev).manual_seed(R)
    grad = torch.randn(W, ld, device=dev, generator=gen).to(dtype)
    arrival = torch.tensor([3.0, 1.0, 2.0, 1.0, float("inf"), 0.5, 9.0], device=dev)
    tags = torch.tensor([4, 4, 4, 4, 4, 3, 4], dtype=torch.int32, device=dev)  # kept: 1, 3, 2, 0, 6
    grad[4] = float("nan")
    grad[5] = float("nan")
    theta = torch.randn(P, device=dev, generator=gen)
    m = torch.randn(P, device=dev, generator=gen)
    opt = sgdb.OrthogonalOpt(lr=0.5, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=1.5)
    mask, order, info = selection_buffers(W, N, dev)
    theta0, m0 = theta.double(), m.double()
    sgdb.sgdb_step_orthogonal(grad, B, R, C, arrival, tags, 4, N, b, theta, m, opt, mask, order, info, workspace(B, R, C, True))
    assert order.cpu().tolist() == [1, 3, 2, 0, 6] and info.cpu().tolist() == [5, 0] and mask.cpu().tolist() == [1, 1, 1, 1, 0, 0, 1]
    g = grad[[1, 3, 2, 0, 6], :P].double().mean(0)
    m_r = 0.9 * m0 + g
    assert rel_err(m.cpu().numpy(), m_r.cpu().numpy()) <= 1e-5
    o = reference((g + 0.9 * m_r if nesterov else m_r).reshape(B, R, C)).reshape(P)
    moved = theta.double() - (1 - 0.5 * 0.1) * theta0
    assert off(moved, -0.75 * o) <= tolerance(min(R, C))
    # selection and mean are those of the separate calls, m is one fused multiply-add of them
    mean = torch.empty(P, device=dev)
    sgdb.sgdb_aggregate(grad, P, N, order, info, mean, ld=ld)
    exact = float(np.float32(0.9)) * m0 + mean.double()  # off the true value by 2^-53 of its terms at most
    assert float((m.double() - exact).abs().max()) <= 2.0 ** -23 * float(exact.abs().max())


def test_step_without_enough_gradients_changes_nothing(cuda_device):
    B, R, C, N, b = 1, 40, 56, 3, 1
    P, dev = R * C, "cuda"
    grad = torch.randn(4, P, device=dev)
    arrival = torch.tensor([1.0, float("inf"), 2.0, 3.0], device=dev)
    tags = torch.tensor([2, 2, 2, 1], dtype=torch.int32, device=dev)
    theta, m = torch.randn(P, device=dev), torch.randn(P, device=dev)
    before = theta.clone(), m.clone()
    mask, order, info = selection_buffers(4, N, dev)
    sgdb.sgdb_step_orthogonal(grad, B, R, C, arrival, tags, 2, N, b, theta, m, sgdb.OrthogonalOpt(), mask, order, info, workspace(B, R, C, True))
    assert info.cpu().tolist() == [2, sgdb.SGDB_ERR_INSUFFICIENT]
    assert torch.equal(theta, before[0]) and torch.equal(m, before[1])
    assert mask.cpu().tolist() == [255] * 4 and order.cpu().tolist() == [-7] * 3


def test_other_stream_back_to_back(cuda_device):
    u = [torch.randn(200, 300, device="cuda") for _ in range(6)]
    out = [torch.empty_like(x) for x in u]
    ws = workspace(1, 200, 300)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for x, y in zip(u, out):
            sgdb.sgdb_orthogonalize(x, y, NS, ws)  # one workspace, calls in stream order
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(u, out):
        z = torch.empty_like(x)
        sgdb.sgdb_orthogonalize(x, z, NS, ws)
        assert torch.equal(y, z)
