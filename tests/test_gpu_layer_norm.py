"""Layer norm forward and backward against the formulas in 64 bits, differences, and refusals.

Tolerances: sums of n terms are taken in fp32 over at most 32 terms per thread and a tree of at most 10 levels (or,
for wide rows, a longer run per thread), so a sum is off by at most about 64 x 2^-24 = 4e-6 of the sum of its terms'
magnitudes; a result is rounded to bf16 by at most 2^-9 of its own size (2^-8 at the foot of a binade)."""
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
EPS = 1e-5
SUM = 1e-5  # 64 x 2^-24 with room for the products' own roundings
HALF_ULP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}

SIZES = [(1, 1), (3, 1023), (5, 7), (1, 8), (4, 64), (33, 96), (9, 128), (130, 256), (70, 768), (17, 1000), (2, 1024), (65, 1025),
         (300, 2048), (3, 4095), (9, 4096), (5, 8192), (3, 8200), (2, 16384), (2, 16392), (2, 20011), (1, 40000), (2000, 64), (5000, 24)]


def rows(T, D, dtype, seed, pad=0, offset=0.0):
    """[T, D] with `pad` elements between the rows' ends and the next rows, guarded by a pattern."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = torch.full((T, D + pad), 77.0, dtype=dtype, device="cuda")
    whole[:, :D] = (torch.randn(T, D, device="cuda", generator=g) + offset).to(dtype)
    return whole, whole[:, :D]


def forward_ref(x, gamma, beta, eps=EPS):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    n = (x - mean[:, None]) * rstd[:, None]
    return n * gamma.double() + beta.double(), mean, rstd, n


def run_forward(T, D, dtype, dt_w, pad=0, offset=0.0, params=True):
    _, x = rows(T, D, dtype, 1, pad, offset)
    whole, y = rows(T, D, dtype, 2, pad)
    gamma = rows(1, D, dt_w, 3)[1].reshape(D) if params else None
    beta = rows(1, D, dt_w, 4)[1].reshape(D) if params else None
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    sgdb.sgdb_layer_norm(x, gamma, beta, EPS, y, mean, rstd)
    one, zero = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    g, b = (gamma, beta) if params else (one, zero)
    y_r, mean_r, rstd_r, n = forward_ref(x, g, b)
    assert bool((whole[:, D:] == 77.0).all())
    mag = x.double().abs().mean(1)
    assert bool(((mean.double() - mean_r).abs() <= SUM * mag + 1e-30).all())
    # rstd: relative, with the mean's error and the roundings of x - mean against the spread
    off = (SUM + 2.0 ** -22 * mag * rstd_r)
    assert bool(((rstd.double() - rstd_r).abs() <= 4 * off * rstd_r).all())
    slack = (4 * off[:, None] * (n.abs() + 1)) * g.double().abs() + SUM * b.double().abs() + HALF_ULP[dtype] * y_r.abs() + 1e-30
    assert bool(((y.double() - y_r).abs() <= slack).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward(cuda_device, T, D, dtype):
    run_forward(T, D, dtype, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("D", [40, 1000, 4096])
def test_forward_strides_parameters_and_offsets(cuda_device, D, pad, dtype):
    run_forward(37, D, dtype, torch.bfloat16, pad=pad)
    run_forward(37, D, dtype, torch.float32, pad=pad, params=False)
    run_forward(5, D, dtype, torch.float32, pad=pad, offset=50.0)


def test_forward_without_statistics_one_parameter_and_special_rows(cuda_device):
    T, D = 6, 512
    x = torch.randn(T, D, device="cuda")
    x[1] = 3.25  # no spread: the numerator is zero
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    gamma = torch.randn(D, device="cuda")
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    sgdb.sgdb_layer_norm(x, gamma, None, EPS, y)
    zero = torch.zeros(D, device="cuda")
    ref = forward_ref(x, gamma, zero)[0]
    assert bool((y[1] == 0).all())
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())  # the row's mean is not a number
    ok = torch.tensor([0, 1, 4, 5], device="cuda")
    assert bool(((y[ok].double() - ref[ok]).abs() <= 1e-4 * (1 + ref[ok].abs())).all())  # other rows do not see them
    sgdb.sgdb_layer_norm(x, gamma, zero, EPS, y2)
    assert torch.equal(y[ok], y2[ok])


def backward_ref(dy, x, gamma, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    n = (x - mean) * rstd
    h = dy * gamma.double()
    dx = rstd * (h - h.mean(1, keepdim=True) - n * (h * n).mean(1, keepdim=True))
    slack = rstd * (h.abs() + h.abs().mean(1, keepdim=True) + n.abs() * (h * n).abs().mean(1, keepdim=True))
    return dx, slack, (dy * n).sum(0), (dy * n).abs().sum(0), dy.sum(0), dy.abs().sum(0)


def run_backward(T, D, dtype, dt_w, dt_g, pad=0, gamma_given=True):
    _, x = rows(T, D, dtype, 1, pad)
    _, dy = rows(T, D, dtype, 2, pad)
    whole, dx = rows(T, D, dtype, 3, pad)
    gamma = rows(1, D, dt_w, 4)[1].reshape(D) if gamma_given else None
    mean = x.float().mean(1)
    rstd = (x.float().var(1, correction=0) + EPS).rsqrt()
    sums = torch.full((2 * D + 2,), 55.0, dtype=dt_g, device="cuda")  # a worker's row: the sums lie one after the other in it
    dgamma, dbeta = sums[1:D + 1], sums[D + 1:2 * D + 1]
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    g = gamma if gamma_given else torch.ones(D, device="cuda")
    dx_r, slack, dg_r, dg_mag, db_r, db_mag = backward_ref(dy, x, g, mean, rstd)
    assert bool((whole[:, D:] == 77.0).all()) and float(sums[0]) == 55.0 and float(sums[-1]) == 55.0
    assert bool(((dx.double() - dx_r).abs() <= SUM * slack + HALF_ULP[dtype] * dx_r.abs() + 1e-30).all())
    assert bool(((dgamma.double() - dg_r).abs() <= SUM * dg_mag + HALF_ULP[dt_g] * dg_r.abs() + 1e-30).all())
    assert bool(((dbeta.double() - db_r).abs() <= SUM * db_mag + HALF_ULP[dt_g] * db_r.abs() + 1e-30).all())
    again = [torch.empty_like(v) for v in (dx, dgamma, dbeta)]
    sgdb.sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, *again, ws)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))  # the same bits every time


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D", SIZES)
def test_backward(cuda_device, T, D, dtype):
    run_backward(T, D, dtype, torch.float32, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("D", [40, 1000, 4096, 9000])
def test_backward_strides_and_types(cuda_device, D, pad, dtype):
    run_backward(37, D, dtype, torch.bfloat16, torch.bfloat16, pad=pad)
    run_backward(37, D, dtype, torch.float32, torch.bfloat16, pad=pad, gamma_given=False)


def test_backward_against_differences(cuda_device):
    """sum(y dy) along a direction, by central differences of the forward kernel.  y is off by about 1e-6, so the sum over
    2100 elements by about 5e-5, and its difference over 2 h = 0.02 by about 2.5e-3; h^2 terms are smaller."""
    T, D, h = 7, 300, 1e-2
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dy, vx = (torch.randn(T, D, device="cuda", generator=gen) for _ in range(3))
    gamma, beta, vg, vb = (torch.randn(D, device="cuda", generator=gen) for _ in range(4))
    mean, rstd, y = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x)

    def loss(dx, dg, db):
        sgdb.sgdb_layer_norm(x + dx * vx, gamma + dg * vg, beta + db * vb, EPS, y, mean, rstd)
        return float((y.double() * dy.double()).sum())

    slopes = [(loss(*(h * e for e in d)) - loss(*(-h * e for e in d))) / (2 * h) for d in ((1, 0, 0), (0, 1, 0), (0, 0, 1))]
    loss(0, 0, 0)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    for slope, grad, v in zip(slopes, (dx, dgamma, dbeta), (vx, vg, vb)):
        assert abs(slope - float((grad.double() * v.double()).sum())) <= 2e-2


def test_one_sum_and_no_sums(cuda_device):
    D = 33
    dbeta = torch.full((D,), 9.0, device="cuda")
    x1 = torch.randn(4, D, device="cuda")
    mean, rstd = x1.mean(1), (x1.var(1, correction=0) + EPS).rsqrt()
    dx, dx2 = torch.empty_like(x1), torch.empty_like(x1)
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(4, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm_backward(x1, x1, None, mean, rstd, dx, None, dbeta, ws)
    sgdb.sgdb_layer_norm_backward(x1, x1, None, mean, rstd, dx2)
    assert torch.equal(dx, dx2)
    assert bool(((dbeta.double() - x1.double().sum(0)).abs() < 1e-5).all())


def test_sums_without_tokens_are_zero(cuda_device):
    D = 40
    dgamma, dbeta = torch.full((D,), 9.0, device="cuda"), torch.full((D,), 9.0, device="cuda")
    nothing, none = torch.empty(0, D, device="cuda"), torch.empty(0, device="cuda")
    sgdb.sgdb_layer_norm(nothing, None, None, EPS, nothing, none, none)
    sgdb.sgdb_layer_norm_backward(nothing, nothing, None, none, none, nothing, dgamma, dbeta)
    assert bool((dgamma == 0).all()) and bool((dbeta == 0).all())


def test_other_stream(cuda_device):
    x = torch.randn(512, 2048, device="cuda")
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sgdb.sgdb_layer_norm(x, None, None, EPS, y)
    torch.cuda.current_stream().wait_stream(s)
    sgdb.sgdb_layer_norm(x, None, None, EPS, y2, stream=torch.cuda.current_stream())
    assert torch.equal(y, y2)
