"""Rows and matrices in 8 bits and the gate against their definitions in 64 bits.

Quantised numbers and scales are exact operations and one rounding: they have to be equal.  The gate's forward pass rounds
silu(g) u, computed in fp32 with errors of a few 2^-24, to 8 bits: a value next to a border may go to the other side, so its
difference from the value in 64 bits is at most half a step (2^-4 of the value in e4m3, 2^-3 in e5m2, or half the smallest step
times the scale) plus 2^-20 of the value.  The backward pass is a product of at most six factors with a relative error of at most
2^-22 each in fp32, and one rounding to the output's type."""
import pytest
import torch

import f8_helpers as f8
from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float8_e4m3fn: (2.0 ** -4, 2.0 ** -10), torch.float8_e5m2: (2.0 ** -3, 2.0 ** -17)}
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def rows_of(R, D, dtype, gen, pad=0):
    """Rows of many sizes, with zeros, infinities and NaN, tiny and huge blocks; `pad` columns of NaN behind each."""
    whole = torch.full((R, D + pad), float("nan"), device="cuda", dtype=dtype)
    x = torch.randn(R, D, device="cuda", generator=gen) * torch.exp2(torch.randint(-20, 20, (R, 1), device="cuda", generator=gen).float())
    x[::7, : min(D, 130)] = 0.0
    if R > 2:
        x[1, D // 2] = float("inf")
        x[2, 0] = float("nan")
        x[2, D - 1] = float("-inf")
    if R > 4:
        x[3] *= 2.0 ** -120
        x[4] = torch.sign(x[4]) * 3e38
    whole[:, :D] = x.to(dtype)
    return whole[:, :D]


SIZES = [(1, 1), (1, 128), (3, 129), (5, 1001), (33, 64), (17, 640), (700, 200), (64, 4097), (5000, 24)]


@pytest.mark.parametrize("fmt", f8.FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,D", SIZES)
def test_quantize(cuda_device, R, D, dtype, fmt):
    gen = torch.Generator(device="cuda").manual_seed(R + D)
    for pad, pad_q in ((0, 0), (1, 3), (8, 16)):
        x = rows_of(R, D, dtype, gen, pad)
        whole = torch.full((R, D + pad_q), 99, dtype=torch.uint8, device="cuda")
        scale = torch.full((R, (D + 127) // 128 + 2), 77, dtype=torch.uint8, device="cuda")
        q, s = whole.view(fmt)[:, :D], scale.view(torch.float8_e8m0fnu)[:, : (D + 127) // 128]
        sgdb.sgdb_quantize(x, q, s)
        want, e = f8.quantized(x, fmt)
        assert f8.same8(q, want) and torch.equal(scale[:, :-2], (e + 127).to(torch.uint8))
        assert bool((whole[:, D:] == 99).all()) and bool((scale[:, -2:] == 77).all())


@pytest.mark.parametrize("fmt", f8.FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,R,C", [(1, 1, 1), (2, 128, 128), (3, 130, 200), (1, 127, 513), (2, 257, 64), (5, 33, 1000)])
def test_quantize_matrices(cuda_device, B, R, C, dtype, fmt):
    gen = torch.Generator(device="cuda").manual_seed(B + R + C)
    for pad, aligned in ((0, True), (3, False)):
        w = rows_of(B * R, C, dtype, gen, pad).unflatten(0, (B, R))
        e8 = lambda *s: sgdb.empty_f8(*s, dtype=fmt, device="cuda") if aligned else torch.empty(s, dtype=fmt, device="cuda")  # noqa: E731
        q, qt = e8(B, R, C), e8(B, C, R)
        scale = torch.empty(B, (R + 127) // 128, (C + 127) // 128, dtype=torch.float8_e8m0fnu, device="cuda")
        sgdb.sgdb_quantize_matrices(w, q, qt, scale)
        want, e = f8.quantized_matrices(w, fmt)
        assert f8.same8(q, want) and f8.same8(qt, want.float().transpose(1, 2))
        assert torch.equal(scale.view(torch.uint8), (e + 127).to(torch.uint8))
        only = torch.empty_like(qt)
        sgdb.sgdb_quantize_matrices(w, None, only, scale)
        assert f8.same8(only, qt)


@pytest.mark.parametrize("fmt", f8.FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,F", [(1, 1), (1, 4096), (3, 129), (40, 96), (33, 1000), (300, 136), (2, 2049)])
def test_gate_and_its_gradient(cuda_device, R, F, dtype, fmt):
    gen = torch.Generator(device="cuda").manual_seed(R + F)
    blocks = (F + 127) // 128
    for pad in (0, 1):
        h = (3.0 * torch.randn(R, 2 * F + pad, device="cuda", generator=gen)).to(dtype)[:, : 2 * F]
        h[0, 0] = 100.0  # sig is 1, and 0
        h[0, F - 1] = -100.0
        if R > 2:
            h[1] = 0.0
            h[2, F // 2] = float("nan")
        e8 = lambda *s: sgdb.empty_f8(*s, dtype=fmt, device="cuda") if pad == 0 else torch.empty(s, dtype=fmt, device="cuda")  # noqa: E731
        new_scale = lambda *s: torch.empty(s, dtype=torch.float8_e8m0fnu, device="cuda")  # noqa: E731
        a, a_scale, h8, h_scale = e8(R, F), new_scale(R, blocks), e8(R, 2, F), new_scale(R, 2, blocks)
        sgdb.sgdb_gate(h, a, a_scale, h8, h_scale)
        want8, e = f8.quantized(h.reshape(R, 2, F), fmt)
        assert f8.same8(h8, want8) and torch.equal(h_scale.view(torch.uint8), (e + 127).to(torch.uint8))
        g, u = h.double().chunk(2, 1)
        want = g / (1 + torch.exp(-g)) * u
        got, s = f8.wide(a, a_scale), a_scale.double().repeat_interleave(128, -1)[:, :F]
        rel, least = HALF_STEP[fmt]
        fine = torch.isfinite(want)
        assert torch.equal(fine, torch.isfinite(got))
        assert bool(((got - want).abs() <= torch.maximum(rel * want.abs(), least * s) + 2.0 ** -20 * want.abs())[fine].all())
        _, ea = f8.quantized(want.float(), fmt)  # scales: the same but next to a border
        off = a_scale.view(torch.uint8).double() - 127 - ea
        assert float(off.abs().max()) <= 1 and int((off != 0).sum()) <= 1 + off.numel() // 100

        da = torch.randn(R, F + pad, device="cuda", generator=gen).to(dtype)[:, :F]
        dh = torch.full((R, 2 * F + pad), 55.0, dtype=dtype, device="cuda")
        sgdb.sgdb_gate_backward(da, h8, h_scale, dh[:, : 2 * F])
        hd = f8.wide(h8, h_scale)
        gd, ud, d = hd[:, 0], hd[:, 1], da.double()
        sig = 1 / (1 + torch.exp(-gd))
        want = torch.cat([d * ud * sig * (1 + gd * (1 - sig)), d * gd * sig], 1)
        # sig (1 + g (1 - sig)) is a sum of two terms that may cancel: its error is relative to the larger
        size = torch.cat([d.abs() * ud.abs() * (sig + (gd * sig * (1 - sig)).abs()), (d * gd * sig).abs()], 1)
        got = dh[:, : 2 * F].double()
        fine = torch.isfinite(want)
        assert torch.equal(fine, torch.isfinite(got))
        assert bool(((got - want).abs() <= 6 * 2.0 ** -22 * size + ROUNDING[dtype] * want.abs() + 2.0 ** -133)[fine].all())
        assert bool((dh[:, 2 * F:] == 55.0).all())


@pytest.mark.parametrize("fmt", f8.FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gate_of_numbers_of_all_sizes(cuda_device, dtype, fmt):
    """Blocks on both sides of what exp(-g) takes without care for its range: the exponent's rounding is 1.5 |g| 2^-24 of the result, the
    exponential, the inverse and three products six times 2^-24 or less."""
    F = 512
    tops = torch.tensor([1.0, 10.0, 59.0, 60.0, 60.5, 87.0, 89.0, 104.0, 300.0], device="cuda")
    g = (tops[:, None] * torch.linspace(-1, 1, F, device="cuda")).to(dtype)
    g[:, ::128] = -tops[:, None].to(dtype)  # in each block
    u = torch.full_like(g, 1.5) * torch.where(torch.arange(F, device="cuda") % 2 == 0, 1.0, 1e20).to(dtype)
    R = g.size(0)
    a, a_scale, h8, h_scale = (new(*s) for new, s in zip(2 * [lambda *s: sgdb.empty_f8(*s, dtype=fmt, device="cuda"),
                                                             lambda *s: sgdb.empty_scale(*s, device="cuda")], [(R, F)] * 2 + [(R, 2, F)] * 2))
    sgdb.sgdb_gate(torch.cat([g, u], 1), a, a_scale, h8, h_scale)
    gd = g.double()
    want = gd / (1 + torch.exp(-gd)) * u.double()
    s = a_scale.double().repeat_interleave(128, -1)[:, :F]
    rel, least = HALF_STEP[fmt]
    bound = torch.maximum(rel * want.abs(), least * s) + (6 + 1.5 * gd.abs()) * 2.0 ** -24 * want.abs()
    assert bool(((f8.wide(a, a_scale) - want).abs() <= bound).all())


def test_gate_gradient_against_differences(cuda_device):
    """(f(h + d) - f(h - d)) / 2d of silu(g) u in 64 bits at the checkpoint's values: an error of d^2 / 6 times the third
    derivative, at most 1e-7 here, and of 1e-16 / d."""
    R, F = 20, 200
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = 2.0 * torch.randn(R, 2 * F, device="cuda", generator=gen)
    a, h8 = sgdb.empty_f8(R, F, device="cuda"), sgdb.empty_f8(R, 2, F, device="cuda")
    a_scale, h_scale = sgdb.empty_scale(R, F, device="cuda"), sgdb.empty_scale(R, 2, F, device="cuda")
    sgdb.sgdb_gate(h, a, a_scale, h8, h_scale)
    da, dh = torch.randn(R, F, device="cuda", generator=gen), torch.empty(R, 2 * F, device="cuda")
    sgdb.sgdb_gate_backward(da, h8, h_scale, dh)
    at = f8.wide(h8, h_scale)
    f = lambda v: (da.double() * v[:, 0] / (1 + torch.exp(-v[:, 0])) * v[:, 1])  # noqa: E731
    for half in (0, 1):
        d = torch.zeros(1, 2, 1, dtype=torch.float64, device="cuda")
        d[0, half] = 1e-4
        want = (f(at + d) - f(at - d)) / 2e-4
        assert float((dh.view(R, 2, F)[:, half].double() - want).abs().max()) <= 2e-6 * float(want.abs().max())


def test_no_rows_and_many_elements(cuda_device):
    for fmt in f8.FORMATS:
        x = torch.empty(0, 64, device="cuda")
        sgdb.sgdb_quantize(x, torch.empty(0, 64, dtype=fmt, device="cuda"), sgdb.empty_scale(0, 64, device="cuda"))
    R, D = 70_000, 32_768  # offsets beyond 32 bits
    x = torch.zeros(R, D, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, D, device="cuda").bfloat16()
    q, s = sgdb.empty_f8(R, D, device="cuda"), sgdb.empty_scale(R, D, device="cuda")
    sgdb.sgdb_quantize(x, q, s)
    want, e = f8.quantized(x[-3:], torch.float8_e4m3fn)
    assert f8.same8(q[-3:], want) and torch.equal(s[-3:].view(torch.uint8), (e + 127).to(torch.uint8)) and not bool(q[: R - 3].view(torch.uint8).any())
