"""The layers' gradients through autograd against the same block written with torch in 64 bits, and the training example."""
import importlib.util
import os

import pytest
import torch

from paper_1604_00981_b200 import layers

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_block_against_torch_in_64_bits(cuda_device):
    """fp32 kernels, sums of at most 96 terms: everything within 1e-5 of the largest value of its tensor."""
    T, D, E, k = 50, 96, 5, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    x, gamma, beta, w, mats = new(2, T // 2, D), new(D), new(D), new(T, k), new(E, D, D) * 0.1
    ids = torch.randint(-1, E, (T, k), device="cuda", generator=gen).int()
    target = new(2, T // 2, D)

    def leaves(dtype):
        return [v.to(dtype).detach().requires_grad_() for v in (x, gamma, beta, w, mats)]

    a = leaves(torch.float32)
    h = layers.layer_norm(a[0], a[1], a[2]).view(T, D)
    r = layers.route(ids, E)
    xs = layers.dispatch(h, r)
    edges = r.offsets.tolist()
    ys = torch.cat([xs[i:j] @ a[4][e] for e, (i, j) in enumerate(zip(edges, edges[1:]))] + [xs[edges[-1]:]])
    out = layers.combine(ys, a[3], r)
    (out * target.view(T, D)).sum().backward()

    c = leaves(torch.float64)
    mean = c[0].mean(-1, keepdim=True)
    var = (c[0] - mean).square().mean(-1, keepdim=True)
    hh = ((c[0] - mean) / torch.sqrt(var + 1e-5) * c[1] + c[2]).view(T, D)
    ref = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    for j in range(k):
        for e in range(E):
            rows = (ids[:, j] == e).nonzero()[:, 0]
            ref = ref.index_add(0, rows, (hh[rows] @ c[4][e]) * c[3][rows, j, None])
    (ref * target.double().view(T, D)).sum().backward()
    assert float((out.double() - ref).detach().abs().max()) <= 1e-5 * float(ref.detach().abs().max())
    for got, want in zip(a, c):
        assert float((got.grad.double() - want.grad).abs().max()) <= 1e-5 * float(want.grad.abs().max())


def test_parameters_that_need_no_gradient(cuda_device):
    x = torch.randn(7, 40, device="cuda").bfloat16().requires_grad_()
    gamma = torch.randn(40, device="cuda")
    layers.layer_norm(x, gamma).float().sum().backward()
    first = x.grad.clone()
    x.grad = None
    layers.layer_norm(x, gamma.requires_grad_()).float().sum().backward()
    assert torch.equal(first, x.grad) and gamma.grad.dtype == torch.float32
    x.grad = None
    layers.layer_norm(x).float().sum().backward()
    assert x.grad is not None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_example_learns(cuda_device, dtype):
    spec = importlib.util.spec_from_file_location("train_experts", os.path.join(ROOT, "examples", "train_experts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=25, dtype=dtype)
    assert losses[-1] < 0.5 * losses[0]  # the successor of each of 32 tokens, from log 32 and more down
