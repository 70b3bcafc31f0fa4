"""Tokens to their experts and back: the sort against a stable sort, copies bit for bit, sums and gradients against 64 bits.

Tolerances: a combined element is a sum of k products in fp32 (k roundings of partial sums and none of the products), a
weight's gradient a sum of `width` products over 32 lanes; rounding to bf16 is at most 2^-8 of the result."""
import numpy as np
import pytest
import torch

from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}


def choices(T, k, E, seed, drop=0.1):
    rng = np.random.Generator(np.random.Philox(seed))
    ids = rng.integers(0, E, (T, k)).astype(np.int32)
    out = rng.random((T, k))
    ids[out < drop / 2] = -1
    ids[out > 1 - drop / 2] = E + rng.integers(0, 5)
    return ids


def route_ref(ids, E):
    flat = ids.reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    used = int((key < E).sum())
    slot = np.full(flat.size, -1, np.int32)
    slot[order[:used]] = np.arange(used)
    source = np.full(flat.size, -1, np.int32)
    source[:used] = order[:used]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])]).astype(np.int32)
    return offsets, slot.reshape(ids.shape), source


def route(ids, E):
    T, k = ids.shape
    dev = torch.from_numpy(ids).cuda()
    offsets = torch.full((E + 1,), -9, dtype=torch.int32, device="cuda")
    slot = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    source = torch.full((T * k,), -9, dtype=torch.int32, device="cuda")
    sgdb.sgdb_route(dev, E, offsets, slot, source)
    return offsets, slot, source


SIZES = [(1, 1, 1), (1, 8, 8), (3, 2, 5), (31, 1, 7), (33, 3, 4), (700, 6, 64), (1024, 4, 256), (1366, 3, 1), (1365, 3, 2), (4096, 1, 1024), (4097, 1, 1000),
         (8192, 8, 64), (5001, 7, 129), (100_000, 2, 16), (3, 32, 40)]


@pytest.mark.parametrize("T,k,E", SIZES)
def test_route(cuda_device, T, k, E):
    for drop in (0.0, 0.3):
        ids = choices(T, k, E, T + k + E, drop)
        got = route(ids, E)
        for g, r in zip(got, route_ref(ids, E)):
            assert np.array_equal(g.cpu().numpy(), r)


@pytest.mark.parametrize("T", [1, 5000])
def test_route_all_dropped_one_expert_and_sorted_input(cuda_device, T):
    E = 10
    for ids in (np.full((T, 2), -1), np.full((T, 2), 2 ** 31 - 1), np.full((T, 2), -(2 ** 31)), np.full((T, 2), 9), np.zeros((T, 2)),
                np.sort(choices(T, 2, E, 1, 0.0).reshape(-1)).reshape(T, 2)):
        ids = ids.astype(np.int32)
        for g, r in zip(route(ids, E), route_ref(ids, E)):
            assert np.array_equal(g.cpu().numpy(), r)


def test_no_tokens(cuda_device):
    e = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    offsets = torch.full((5,), 7, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 16, device="cuda")
    w = torch.empty(0, 2, device="cuda")
    sgdb.sgdb_route(e, 4, offsets, e, e.reshape(0))
    assert offsets.cpu().tolist() == [0] * 5
    sgdb.sgdb_dispatch(x, e, offsets, x)
    sgdb.sgdb_combine(x, e, w, x)
    sgdb.sgdb_combine_backward(x, x, e, w, offsets, x, w)


def guarded(rows, D, dtype, pad, gen=None):
    whole = torch.full((rows, D + pad), 77.0, dtype=dtype, device="cuda")
    if gen is not None:
        whole[:, :D] = torch.randn(rows, D, device="cuda", generator=gen).to(dtype)
    return whole, whole[:, :D]


CASES = [(1, 1, 1, 1), (1, 8192, 8, 8), (5, 7, 2, 3), (40, 64, 3, 8), (33, 1000, 2, 16), (129, 1001, 1, 4), (64, 2048, 8, 64), (17, 4104, 4, 5),
         (3000, 16, 2, 32), (2, 130, 32, 50)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [0, 1, 8])
@pytest.mark.parametrize("T,D,k,E", CASES)
def test_dispatch_combine_and_gradients(cuda_device, T, D, k, E, pad, dtype):
    gen = torch.Generator(device="cuda").manual_seed(T * 7 + D)
    ids = choices(T, k, E, 3, 0.2)
    ids[0] = -1  # a token that no expert takes
    offsets, slot, source = route(ids, E)
    used = int(offsets[-1])
    src = source[:used].long()
    _, x = guarded(T, D, dtype, pad, gen)
    wxs, xs = guarded(T * k, D, dtype, pad)
    sgdb.sgdb_dispatch(x, slot, offsets, xs)
    assert torch.equal(xs[:used], x[src // k]) and bool((xs[used:] == 0).all()) and bool((wxs[:, D:] == 77.0).all())

    _, ys = guarded(T * k, D, dtype, pad, gen)
    ys[used:] = float("nan")  # rows that belong to no pair are never read
    w = torch.randn(T, k, device="cuda", generator=gen)
    w[slot < 0] = float("nan")  # nor do the weights of dropped pairs matter
    wout, out = guarded(T, D, dtype, pad)
    terms = ys[:used].double() * w.double().reshape(-1)[src][:, None]
    zero = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    ref, mag = zero.index_add(0, src // k, terms), zero.index_add(0, src // k, terms.abs())
    sgdb.sgdb_combine(ys, slot, w, out)
    assert bool((wout[:, D:] == 77.0).all()) and bool((out[0] == 0).all())
    assert bool(((out.double() - ref).abs() <= (k + 1) * 2.0 ** -24 * mag + HALF_ULP[dtype] * ref.abs()).all())
    sgdb.sgdb_combine(ys, slot, None, out)  # the gradient of dispatch
    terms = ys[:used].double()
    ref, mag = zero.index_add(0, src // k, terms), zero.index_add(0, src // k, terms.abs())
    assert bool(((out.double() - ref).abs() <= (k + 1) * 2.0 ** -24 * mag + HALF_ULP[dtype] * ref.abs()).all())

    _, dout = guarded(T, D, dtype, pad, gen)
    wdys, dys = guarded(T * k, D, dtype, pad)
    dw = torch.full((T, k), 5.0, device="cuda")
    sgdb.sgdb_combine_backward(dout, ys, slot, w, offsets, dys, dw)
    ref = dout.double()[src // k] * w.double().reshape(-1)[src][:, None]
    assert bool(((dys[:used].double() - ref).abs() <= 2 * HALF_ULP[dtype] * ref.abs()).all())
    assert bool((dys[used:] == 0).all()) and bool((wdys[:, D:] == 77.0).all())
    prod = dout.double()[src // k] * ys[:used].double()
    flat = dw.double().reshape(-1)
    assert bool(((flat[src] - prod.sum(1)).abs() <= (D / 32 + 8) * 2.0 ** -24 * prod.abs().sum(1) + 1e-30).all())
    assert bool((dw[slot < 0] == 0).all())
    dys2 = torch.empty_like(dys)
    sgdb.sgdb_combine_backward(dout, ys, slot, None, offsets, dys2)
    assert torch.equal(dys2[:used], dout[src // k])


def test_gradients_against_differences(cuda_device):
    """combine is linear in ys and in w: one difference along a direction is exact up to the roundings of the two sums
    (T D = 640 elements, each off by about 2e-7)."""
    T, D, k, E = 20, 32, 3, 6
    gen = torch.Generator(device="cuda").manual_seed(1)
    offsets, slot, source = route(choices(T, k, E, 9, 0.2), E)
    ys, vy = (torch.randn(T * k, D, device="cuda", generator=gen) for _ in range(2))
    w, vw = (torch.randn(T, k, device="cuda", generator=gen) for _ in range(2))
    dout = torch.randn(T, D, device="cuda", generator=gen)
    out = torch.empty(T, D, device="cuda")

    def loss(a, b):
        sgdb.sgdb_combine(ys + a * vy, slot, w + b * vw, out)
        return float((out.double() * dout.double()).sum())

    dys, dw = torch.empty_like(ys), torch.empty_like(w)
    sgdb.sgdb_combine_backward(dout, ys, slot, w, offsets, dys, dw)
    assert abs(loss(0.5, 0) - loss(-0.5, 0) - float((dys.double() * vy.double()).sum())) < 1e-3
    assert abs(loss(0, 0.5) - loss(0, -0.5) - float((dw.double() * vw.double()).sum())) < 1e-3


def test_slots_out_of_range_are_dropped(cuda_device):
    T, D, k = 4, 24, 2
    x = torch.randn(T, D, device="cuda")
    slot = torch.tensor([[0, 8], [1, -5], [2 ** 31 - 1, 2], [-(2 ** 31), 7]], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    whole = torch.full((T * k + 2, D), 3.0, device="cuda")
    sgdb.sgdb_dispatch(x, slot, offsets, whole[1:-1])
    xs = whole[1:-1]
    assert torch.equal(xs[0], x[0]) and torch.equal(xs[1], x[1]) and torch.equal(xs[2], x[2]) and torch.equal(xs[7], x[3])
    assert bool((xs[3:7] == 3.0).all()) and bool((whole[0] == 3.0).all()) and bool((whole[-1] == 3.0).all())
    out = torch.empty_like(x)
    sgdb.sgdb_combine(xs, slot, None, out)
    assert torch.equal(out, x)


def test_rows_beyond_32_bits(cuda_device):
    """Offsets of more than 2^32 bytes and 2^31 elements: the last row of a large buffer."""
    T, D, k = 70_000, 32_768, 1
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(D, device="cuda").remainder(251).bfloat16()
    xs = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    offsets, slot, source = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (2, T, T))
    slot = slot.reshape(T, 1)
    sgdb.sgdb_route(ids, 1, offsets, slot, source)
    sgdb.sgdb_dispatch(x, slot, offsets, xs)
    assert torch.equal(xs[-1], x[-1]) and int(xs[:-1].count_nonzero()) == 0
    out = x.zero_()
    sgdb.sgdb_combine(xs, slot, torch.full((T, 1), 2.0, device="cuda"), out)
    assert torch.equal(out[-1], xs[-1] * 2)
