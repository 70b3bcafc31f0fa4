"""Layer norm backward of rows that do not fill their chunks: columns beyond the row's end have no part in its sums, however
large mean * rstd is."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("D", [4, 8, 100, 264, 700, 1000, 2056, 4096, 4500, 8190])
def test_equal_columns_whose_mean_times_rstd_overflows(cuda_device, D, pad, dtype):
    """A row of one value has n = 0 and rstd = 1 / sqrt(eps): dx = rstd (dy - mean(dy)), dgamma = 0, dbeta = dy.  The mean given
    is the value itself, so nothing is rounded before the mean of dy, a sum of at most D terms (1e-5 of their magnitudes)."""
    value, eps = 2.0 ** 110, 1e-12
    T = 3
    gen = torch.Generator(device="cuda").manual_seed(D)
    x = torch.full((T, D + pad), value, device="cuda").to(dtype)[:, :D]
    dy = torch.randn(T, D + pad, device="cuda", generator=gen).to(dtype)[:, :D]
    mean = torch.full((T,), value, device="cuda")
    rstd = torch.full((T,), eps ** -0.5, device="cuda")
    dx = torch.empty(T, D + pad, dtype=dtype, device="cuda")[:, :D]
    dgamma, dbeta = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm_backward(dy, x, None, mean, rstd, dx, dgamma, dbeta, ws)
    d = dy.double()
    want = (d - d.mean(1, keepdim=True)) * float(rstd[0])
    slack = 1e-5 * float(rstd[0]) * (d.abs() + d.abs().mean(1, keepdim=True)) + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * want.abs()
    assert bool(((dx.double() - want).abs() <= slack).all())
    assert bool((dgamma == 0).all())
    assert bool(((dbeta.double() - d.sum(0)).abs() <= 1e-5 * d.abs().sum(0)).all())
