"""The layers in bf16 and fp32, with parameters of either type: outputs and gradients are those of the binding's calls, bit for
bit, and of the types of their tensors.  (The calls themselves are held to 64 bits in their own tests.)"""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb
from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu


def grads(y, leaves, dy):
    return torch.autograd.grad(y, leaves, dy)


@pytest.mark.parametrize("dt_w", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D", [(1, 1), (37, 96), (20, 333), (300, 2048)])
def test_layer_norm(cuda_device, T, D, dtype, dt_w):
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, dy = (torch.randn(T, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    gamma, beta = (torch.randn(D, device="cuda", generator=gen).to(dt_w) for _ in range(2))
    leaves = [v.clone().requires_grad_() for v in (x, gamma, beta)]
    got = layers.layer_norm(*leaves)
    got = [got.detach(), *grads(got, leaves, dy)]
    want = [torch.empty_like(v) for v in (x, x, gamma, beta)]
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm(x, gamma, beta, 1e-5, want[0], mean, rstd)
    sgdb.sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, *want[1:], ws)
    assert all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D,k,E", [(1, 1, 1, 1), (37, 96, 2, 5), (20, 333, 3, 8), (300, 2048, 2, 16)])
def test_experts(cuda_device, T, D, k, E, dtype):
    gen = torch.Generator(device="cuda").manual_seed(D)
    ids = torch.randint(-1, E + 1, (T, k), device="cuda", generator=gen).int()
    r = layers.route(ids, E)
    x, dout = (torch.randn(T, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    ys, dxs = (torch.randn(T * k, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    w = torch.randn(T, k, device="cuda", generator=gen)
    lx, ly, lw = (v.clone().requires_grad_() for v in (x, ys, w))
    xs, out, plain = layers.dispatch(lx, r), layers.combine(ly, lw, r), layers.combine(ly, None, r)
    got = [xs.detach(), *grads(xs, [lx], dxs), out.detach(), *grads(out, [ly, lw], dout), plain.detach(), *grads(plain, [ly], dout)]
    want = [torch.empty_like(v) for v in (ys, x, x, ys, w, x, ys)]
    sgdb.sgdb_dispatch(x, r.slot, r.offsets, want[0])
    sgdb.sgdb_combine(dxs, r.slot, None, want[1])
    sgdb.sgdb_combine(ys, r.slot, w, want[2])
    sgdb.sgdb_combine_backward(dout, ys, r.slot, w, r.offsets, want[3], want[4])
    sgdb.sgdb_combine(ys, r.slot, None, want[5])
    sgdb.sgdb_combine_backward(dout, ys, r.slot, None, r.offsets, want[6])
    assert all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, want))
