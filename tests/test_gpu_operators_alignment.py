"""The worker's operators on arrays that begin anywhere: every element offset against 16-byte boundaries, alike and
different from array to array.  Copies have to be equal bit for bit; layer norm is held to the same call on aligned copies of
its inputs, whose sums over columns are taken in another order (at most 64 x 2^-24 of the sum of magnitudes)."""
import itertools

import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def at_offset(values, off):
    """`values` in memory that begins `off` elements after a 16-byte boundary, and the whole buffer with a guard around them."""
    n = values.numel()
    whole = torch.full((n + 32,), 77.0, dtype=values.dtype, device="cuda") if values.is_floating_point() else \
        torch.full((n + 32,), -77, dtype=values.dtype, device="cuda")
    view = whole[8 + off:8 + off + n].view(values.shape)
    view.copy_(values)
    return whole, view


def untouched(whole, off, n):
    return bool((whole[:8 + off] == 77.0).all()) and bool((whole[8 + off + n:] == 77.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D", [(1, 5), (19, 40), (70, 333), (33, 1000), (21, 4101)])
def test_layer_norm(cuda_device, T, D, dtype):
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, dy = (torch.randn(T, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    gamma, beta = (torch.randn(D, device="cuda", generator=gen) for _ in range(2))
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(sgdb.sgdb_layer_norm_backward_workspace_bytes(T, D), dtype=torch.uint8, device="cuda")
    sgdb.sgdb_layer_norm(x, gamma, beta, 1e-5, y, mean, rstd)
    sgdb.sgdb_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, ws)
    n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    h = dy.double() * gamma.double()
    slack_y = 1e-5 * (n.abs() + 1) * gamma.abs() + 1e-5 * beta.abs() + 2 * HALF_ULP[dtype] * y.double().abs()
    slack_dx = 1e-5 * rstd.double()[:, None] * (h.abs() + h.abs().mean(1, keepdim=True) + n.abs() * (h * n).abs().mean(1, keepdim=True)) \
        + 2 * HALF_ULP[dtype] * dx.double().abs()
    for a, b, c in ((0, 0, 0), (1, 1, 1), (3, 3, 3), (1, 1, 0), (2, 2, 3), (0, 1, 0), (3, 0, 2)):  # x, dy, output
        m2, r2 = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        xo, dyo = at_offset(x, a)[1], at_offset(dy, b)[1]
        whole, yo = at_offset(torch.zeros_like(y), c)
        sgdb.sgdb_layer_norm(xo, gamma, beta, 1e-5, yo, m2, r2)
        assert untouched(whole, c, T * D)
        assert bool(((yo.double() - y.double()).abs() <= slack_y).all())
        whole, dxo = at_offset(torch.zeros_like(dx), c)
        dg2, db2 = at_offset(torch.zeros_like(dg), 1)[1], at_offset(torch.zeros_like(db), 3)[1]
        sgdb.sgdb_layer_norm_backward(dyo, xo, gamma, mean, rstd, dxo, dg2, db2, ws)
        assert untouched(whole, c, T * D)
        assert bool(((dxo.double() - dx.double()).abs() <= slack_dx).all())
        assert bool(((dg2 - dg).double().abs() <= 1e-5 * (dy.double() * n).abs().sum(0)).all())
        assert bool(((db2 - db).double().abs() <= 1e-5 * dy.double().abs().sum(0)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,D,k", [(1, 3, 1), (9, 24, 2), (13, 517, 3), (6, 2056, 4)])
def test_experts(cuda_device, T, D, k, dtype):
    E = 4
    gen = torch.Generator(device="cuda").manual_seed(D)
    ids = torch.randint(-1, E + 1, (T, k), device="cuda", generator=gen).int()
    new = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets, slot, source = new(E + 1), new(T, k), new(T * k)
    sgdb.sgdb_route(ids, E, offsets, slot, source)
    for off in (1, 2, 3):
        o2, s2, r2 = (at_offset(v, 4 - off)[1] for v in (torch.zeros_like(offsets), torch.zeros_like(slot), torch.zeros_like(source)))
        sgdb.sgdb_route(at_offset(ids, off)[1], E, o2, s2, r2)
        assert torch.equal(o2, offsets) and torch.equal(s2, slot) and torch.equal(r2, source)
    used = int(offsets[-1])
    x, dout = (torch.randn(T, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    ys = torch.randn(T * k, D, device="cuda", generator=gen).to(dtype)
    w = torch.randn(T, k, device="cuda", generator=gen)
    out, dys, dw = torch.empty_like(x), torch.empty_like(ys), torch.empty_like(w)
    sgdb.sgdb_combine(ys, slot, w, out)
    sgdb.sgdb_combine_backward(dout, ys, slot, w, offsets, dys, dw)
    mag = torch.zeros(T * k, dtype=torch.float64, device="cuda")
    src = source[:used].long()
    mag[src] = (dout.double()[src // k] * ys[:used].double()).abs().sum(1)
    per = 4 if dtype == torch.float32 else 8
    for a, b in itertools.product(range(0, per, 3 if per == 8 else 1), (0, 1, per - 1)):
        whole, xs = at_offset(torch.zeros_like(ys), b)
        sgdb.sgdb_dispatch(at_offset(x, a)[1], slot, offsets, xs)
        assert untouched(whole, b, ys.numel())
        assert torch.equal(xs[:used], x[src // k]) and bool((xs[used:] == 0).all())
        whole, out2 = at_offset(torch.zeros_like(out), b)
        sgdb.sgdb_combine(at_offset(ys, a)[1], slot, w, out2)
        assert untouched(whole, b, out.numel()) and torch.equal(out2, out)  # the same sums in the same order
        whole, dys2 = at_offset(torch.zeros_like(dys), b)
        dw2 = torch.zeros_like(dw)
        sgdb.sgdb_combine_backward(at_offset(dout, a)[1], at_offset(ys, (a + b) % per)[1], slot, w, offsets, dys2, dw2)
        assert untouched(whole, b, dys.numel()) and torch.equal(dys2, dys)
        assert bool(((dw2 - dw).double().abs().reshape(-1) <= (D / 32 + 16) * 2.0 ** -23 * mag).all())
