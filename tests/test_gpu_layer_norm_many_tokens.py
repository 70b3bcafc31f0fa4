"""Layer norm backward over many tokens whose dy begins otherwise against 16-byte boundaries than x: the sums of dgamma and dbeta.

A thread adds T / 592 rows (592 partial sums, as many as the workspace has room for from 592 x 32 rows on), the second kernel
37 partial sums per warp and 16 warps: a sum is off by at most (T / 592 + 64) x 2^-24 of its terms' magnitudes.  dy is one
value, chosen so that the additions to a running sum above 2048 all round the same way."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,D", [(1 << 18, 8), (1 << 18, 5), (300_000, 64)])
def test_sums_over_many_tokens(cuda_device, T, D):
    value = 1.0 + 0.99 * 2.0 ** -13
    x = torch.randn(T, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    dy = torch.full((T * D + 1,), value, device="cuda")[1:].view(T, D)
    mean = x.mean(1)
    rstd = (x.var(1, correction=0) + 1e-5).rsqrt()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm_backward(dy, x, None, mean, rstd, dx, dgamma, dbeta, ws)
    n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    bound = (T / 592 + 64) * 2.0 ** -24
    assert bool(((dbeta.double() - dy.double().sum(0)).abs() <= bound * dy.double().sum(0)).all())
    assert bool(((dgamma.double() - (dy.double() * n).sum(0)).abs() <= bound * (dy.double() * n).abs().sum(0)).all())
    want = rstd.double()[:, None] * (dy.double() - dy.double().mean(1, keepdim=True) - n * (dy.double() * n).mean(1, keepdim=True))
    slack = rstd.double()[:, None] * (dy.double() * 2 + n.abs() * (dy.double() * n).abs().mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= 1e-5 * slack).all())
