"""The experts' products of 8-bit rows and matrices, and their matrices' gradient, against 64 bits.

Products of 8-bit numbers are exact in fp32; sums in tensor memory lose at most a bit of 2^-23 of the running sum at each of the
K / 32 instructions and inside each: an error of (K / 32 + 8) 2^-23 of the sum of magnitudes covers it.  The gradient with dy
in bf16 adds 16 tokens at a time: (tokens / 16 + 8) 2^-23; with dy in fp32 it is cut into three exact parts whose sums over 64 tokens
are added with 2^-24 each: (12 + 8 + tokens / 64) 2^-23."""
import pytest
import torch

import f8_helpers as f8
from paper_1604_00981_b200 import binding as sgdb

pytestmark = pytest.mark.gpu
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def eight_bit(rows, cols, fmt, gen, spread=3):
    """Rows in 8 bits with scales of many sizes, as sgdb_quantize's caller would hold them."""
    x = torch.randn(rows, cols, device="cuda", generator=gen) * torch.exp2(torch.randint(-spread, spread + 1, (rows, 1), device="cuda", generator=gen).float())
    q, e = f8.quantized(x, fmt)
    out, scale = sgdb.empty_f8(rows, cols, dtype=fmt, device="cuda"), sgdb.empty_scale(rows, cols, device="cuda")
    out.copy_(q)
    scale.copy_(f8.scales(e))
    return out, scale


def matrices(E, N, K, fmt, gen):
    w = torch.randn(E, N, K, device="cuda", generator=gen)
    q, qt = sgdb.empty_f8(E, N, K, dtype=fmt, device="cuda"), sgdb.empty_f8(E, K, N, dtype=fmt, device="cuda")
    scale = torch.empty(E, (N + 127) // 128, (K + 127) // 128, dtype=torch.float8_e8m0fnu, device="cuda")
    sgdb.sgdb_quantize_matrices(w, q, qt, scale)
    return q, qt, scale


def offsets_of(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32, device="cuda")


def by_expert(counts):
    at = 0
    for e, n in enumerate(counts):
        yield e, slice(at, at + n)
        at += n


# rows of each expert, rows not in use, width, depth
CASES = [
    ([1], 0, 1, 1), ([1], 0, 256, 128), ([0, 1, 0], 2, 70, 200), ([5, 0, 17, 1], 0, 130, 600), ([240], 0, 256, 512), ([241, 16, 3], 5, 300, 130),
    ([33, 480, 7], 1, 129, 2048), ([1] * 8 + [0] * 56, 0, 512, 640), ([1000], 24, 1001, 500), ([0, 0], 9, 64, 64), ([600, 700], 0, 768, 1408),
    ([3] * 300, 0, 40, 100), ([100, 200, 300], 0, 2816, 4224),
]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_product(cuda_device, case, dt):
    counts, unused, N, K = CASES[case]
    S, E = sum(counts) + unused, len(counts)
    for fx, fw in ((torch.float8_e4m3fn, torch.float8_e4m3fn), (torch.float8_e5m2, torch.float8_e4m3fn), (torch.float8_e4m3fn, torch.float8_e5m2)):
        gen = torch.Generator(device="cuda").manual_seed(case)
        x, xs = eight_bit(S, K, fx, gen)
        w, wt, ws = matrices(E, N, K, fw, gen)
        if unused:
            x[S - unused:].view(torch.uint8).fill_(0x7f)  # NaN in rows that belong to nobody
        whole = torch.full((S + 2, N + 8), 77.0, dtype=dt, device="cuda")
        y = whole[1:-1, :N]
        info = torch.zeros(2, dtype=torch.int32, device="cuda")
        sgdb.sgdb_experts_product(x, xs, w, ws, offsets_of(counts), y, info)
        assert info.tolist() == [0, 0]
        xd, wd = f8.wide(x, xs), f8.wide_matrices(w, ws)
        for e, rows in by_expert(counts):
            want, size = xd[rows] @ wd[e].T, xd[rows].abs() @ wd[e].abs().T
            assert bool(((y[rows].double() - want).abs() <= (K / 32 + 8) * 2.0 ** -23 * size + ROUNDING[dt] * want.abs()).all())
        assert unused == 0 or not bool(y[S - unused:].any())
        assert bool((whole[0] == 77.0).all()) and bool((whole[-1] == 77.0).all()) and bool((whole[:, N:] == 77.0).all())
        # the matrices' other direction: the gradient of the rows
        if K <= 2048:
            dy, dys = eight_bit(S, N, fx, gen)
            dx = torch.empty(S, K, dtype=dt, device="cuda")
            sgdb.sgdb_experts_product(dy, dys, wt, ws.transpose(1, 2), offsets_of(counts), dx)
            dd = f8.wide(dy, dys)
            for e, rows in by_expert(counts):
                want, size = dd[rows] @ wd[e], dd[rows].abs() @ wd[e].abs()
                assert bool(((dx[rows].double() - want).abs() <= (N / 32 + 8) * 2.0 ** -23 * size + ROUNDING[dt] * want.abs()).all())


def test_a_bad_row_stays_by_itself(cuda_device):
    """NaN in one row, in a scale, in one expert's matrix: nobody else's results change."""
    counts, N, K = [70, 50, 30], 200, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, xs = eight_bit(150, K, torch.float8_e4m3fn, gen)
    w, _, ws = matrices(3, N, K, torch.float8_e4m3fn, gen)
    off = offsets_of(counts)
    want, got = torch.empty(150, N, device="cuda"), torch.empty(150, N, device="cuda")
    sgdb.sgdb_experts_product(x, xs, w, ws, off, want)
    x[69].view(torch.uint8)[5] = 0x7f
    xs[3].view(torch.uint8)[2] = 255
    ws[2].view(torch.uint8).fill_(255)
    sgdb.sgdb_experts_product(x, xs, w, ws, off, got)
    bad = torch.zeros(150, dtype=torch.bool, device="cuda")
    bad[[69, 3]] = True
    bad[120:] = True
    assert bool(got[bad].isnan().all()) and torch.equal(got[~bad], want[~bad])


def test_one_expert_without_offsets_any_strides(cuda_device):
    gen = torch.Generator(device="cuda").manual_seed(2)
    S, N, K = 100, 96, 256
    x, xs = eight_bit(S, K, torch.float8_e4m3fn, gen)
    w, _, ws = matrices(1, N, K, torch.float8_e4m3fn, gen)
    want, got = torch.empty(S, N, device="cuda"), torch.empty(S, N, device="cuda")
    sgdb.sgdb_experts_product(x, xs, w, ws, offsets_of([S]), want)
    wide_x = torch.empty(S, K + 32, dtype=x.dtype, device="cuda")
    wide_x[:, 16:-16] = x
    odd_scale = torch.empty(S, 3, dtype=xs.dtype, device="cuda")
    odd_scale[:, 1:] = xs
    sgdb.sgdb_experts_product(wide_x[:, 16:-16], odd_scale[:, 1:], w, ws, None, got)  # scales on no boundary at all
    assert torch.equal(got, want)
    with pytest.raises(ValueError):
        sgdb.sgdb_experts_product(x, xs, w, ws, offsets_of([S, 0]), got)
    with pytest.raises(sgdb.SgdbError):  # rows that do not begin on 16-byte boundaries
        sgdb.sgdb_experts_product(torch.empty(S, K + 8, dtype=x.dtype, device="cuda")[:, :K], xs, w, ws, None, got)


def test_offsets_that_do_not_rise_stay_in_bounds(cuda_device):
    gen = torch.Generator(device="cuda").manual_seed(2)
    S, N, K = 64, 96, 128
    x, xs = eight_bit(S, K, torch.float8_e4m3fn, gen)
    w, _, ws = matrices(3, N, K, torch.float8_e4m3fn, gen)
    dy, dw = torch.randn(S, N, device="cuda", generator=gen), torch.empty(3, N, K, device="cuda")
    for bad in ([0, 200, -5, 64], [-100, 10, 5, 1000], [64, 0, 64, 0], [2 ** 31 - 1] * 4, [-(2 ** 31)] * 4):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        whole = torch.full((S + 2, N), 77.0, device="cuda")
        sgdb.sgdb_experts_product(x, xs, w, ws, off, whole[1:-1])
        sgdb.sgdb_experts_gradient(dy, x, xs, off, dw)
        assert bool((whole[[0, -1]] == 77.0).all())


def test_offsets_of_elements_beyond_32_bits(cuda_device):
    S, N, K = 140_000, 16_384, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, xs = eight_bit(S, K, torch.float8_e4m3fn, gen)
    w, _, ws = matrices(2, N, K, torch.float8_e4m3fn, gen)
    y = torch.empty(S, N, dtype=torch.bfloat16, device="cuda")
    sgdb.sgdb_experts_product(x, xs, w, ws, offsets_of([S // 2, S // 2 - 7]), y)
    rows = torch.tensor([0, S // 2 - 1, S // 2, S - 8], device="cuda")
    want = torch.stack([f8.wide(x[r][None], xs[r][None])[0] @ f8.wide_matrices(w, ws)[int(r >= S // 2)].T for r in rows])
    assert bool(((y[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * want.abs().max()).all()) and not bool(y[-7:].any())


GRADIENT_CASES = CASES + [([9000], 3, 64, 48), ([30_000, 11], 0, 300, 200), ([64, 128, 65, 63], 0, 512, 256)]


@pytest.mark.parametrize("dt,dt_dw", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("case", range(len(GRADIENT_CASES)))
def test_gradient(cuda_device, case, dt, dt_dw):
    counts, unused, N, K = GRADIENT_CASES[case]
    S, E = sum(counts) + unused, len(counts)
    for fmt, pad in ((torch.float8_e4m3fn, 0), (torch.float8_e5m2, 1)):
        gen = torch.Generator(device="cuda").manual_seed(case)
        x, xs = eight_bit(S, K, fmt, gen)
        dy = torch.randn(S, N + pad, device="cuda", generator=gen).to(dt)[:, :N]
        if unused:
            dy[S - unused:] = float("nan")
            x[S - unused:].view(torch.uint8).fill_(0x7f)
            xs[S - unused:].view(torch.uint8).fill_(255)
        whole = torch.full((E, N + 1, K + 8 * pad), 77.0, dtype=dt_dw, device="cuda")
        dw = whole[:, :N, :K]
        need = sgdb.sgdb_experts_gradient_workspace_bytes(S, N, K, E)
        info = torch.zeros(2, dtype=torch.int32, device="cuda")
        sgdb.sgdb_experts_gradient(dy, x, xs, offsets_of(counts), dw, torch.empty(need, dtype=torch.uint8, device="cuda"), info)
        assert info.tolist() == [0, 0]
        xd, d = f8.wide(x, xs), dy.double()
        for e, rows in by_expert(counts):
            want, size = d[rows].T @ xd[rows], d[rows].abs().T @ xd[rows].abs()
            steps = 20 + counts[e] / 64 if dt == torch.float32 else 8 + counts[e] / 16
            assert bool(((dw[e].double() - want).abs() <= steps * 2.0 ** -23 * size + ROUNDING[dt_dw] * want.abs()).all())
        assert bool((whole[:, N:] == 77.0).all()) and bool((whole[:, :, K:] == 77.0).all())


def test_gradient_of_others_rows_that_are_not_numbers(cuda_device):
    """Experts share slots of 64 rows: what the neighbours hold does not come through, whatever it is."""
    counts, N, K = [40, 10, 100], 72, 144
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, xs = eight_bit(150, K, torch.float8_e4m3fn, gen)
    for dt in (torch.float32, torch.bfloat16):
        dy = torch.randn(150, N, device="cuda", generator=gen).to(dt)
        want, got = torch.empty(3, N, K, device="cuda"), torch.empty(3, N, K, device="cuda")
        sgdb.sgdb_experts_gradient(dy, x, xs, offsets_of(counts), want)
        bad, bad_x, bad_xs = dy.clone(), x.clone(), xs.clone()
        bad[40:50] = float("inf")
        bad[45] = float("nan")
        bad_x[40:50].view(torch.uint8).fill_(0x7f)
        bad_xs[42].view(torch.uint8).fill_(255)
        sgdb.sgdb_experts_gradient(bad, bad_x, bad_xs, offsets_of(counts), got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and bool(got[1].isnan().all())


def test_gradient_with_a_workspace_on_any_word(cuda_device):
    """Ranges' sums in a workspace that begins on a multiple of 4 bytes only: the bits of an aligned one."""
    S, N, K = 4000, 70, 100
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, xs = eight_bit(S, K, torch.float8_e4m3fn, gen)
    need = sgdb.sgdb_experts_gradient_workspace_bytes(S, N, K, 1)
    assert need > 4
    for dt in (torch.float32, torch.bfloat16):
        dy = torch.randn(S, N, device="cuda", generator=gen).to(dt)
        out = [torch.empty(1, N, K, device="cuda") for _ in range(3)]
        for i, dw in enumerate(out):
            work = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
            sgdb.sgdb_experts_gradient(dy, x, xs, None, dw, work[4 * i:4 * i + need])
        assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


@pytest.mark.parametrize("fmt", f8.FORMATS)
def test_gradient_with_scales_at_both_ends(cuda_device, fmt):
    """Scales from the smallest to the largest that a quantised number has, and infinities of e5m2."""
    S, N, K = 64, 16, 256
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, xs = eight_bit(S, K, fmt, gen)
    xs.view(torch.uint8)[:, 0] = torch.randint(17, 230, (S,), device="cuda", generator=gen).to(torch.uint8)
    dy = torch.zeros(S, N, device="cuda").bfloat16()
    dy[torch.arange(N, device="cuda") * 4, torch.arange(N, device="cuda")] = 1.0  # each result is one element of x
    dw = torch.empty(1, N, K, device="cuda")
    sgdb.sgdb_experts_gradient(dy, x, xs, None, dw)
    assert torch.equal(dw[0].double(), f8.wide(x, xs)[::4][:N])
    if fmt == torch.float8_e5m2:
        x[0].view(torch.uint8)[3] = 0x7c
        sgdb.sgdb_experts_gradient(dy[:, :1], x, xs, None, dw[:, :1])
        assert bool(torch.isinf(dw[0, 0, 3])) and bool(torch.isfinite(dw[0, 0, 4:]).all())


LIMITS_NS = [0, 0, 1, 1_000, 10_000, 100_000]


@pytest.mark.parametrize("counts,N,K", [([40], 96, 2048), ([300, 500], 512, 1408), ([2000] * 4, 1024, 1024)])
def test_waits_that_run_out(cuda_device, counts, N, K):
    """With little patience the kernels end normally and say so; the next call gives the bits that it gave before."""
    S, E = sum(counts), len(counts)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, xs = eight_bit(S, K, torch.float8_e4m3fn, gen)
    w, _, ws = matrices(E, N, K, torch.float8_e4m3fn, gen)
    off, info = offsets_of(counts), torch.zeros(2, dtype=torch.int32, device="cuda")
    work = torch.empty(sgdb.sgdb_experts_gradient_workspace_bytes(S, N, K, E), dtype=torch.uint8, device="cuda")

    def calls():
        for dt in (torch.bfloat16, torch.float32):
            dy = torch.ones(S, N, dtype=dt, device="cuda")
            yield torch.empty(E, N, K, dtype=dt, device="cuda"), lambda out, dy=dy: sgdb.sgdb_experts_gradient(dy, x, xs, off, out, work, info)
            yield torch.empty(S, N, dtype=dt, device="cuda"), lambda out: sgdb.sgdb_experts_product(x, xs, w, ws, off, out, info)

    try:
        for want, call in calls():
            call(want)
            assert info.tolist() == [0, 0]
            for limit in LIMITS_NS:
                sgdb.sgdb_set_wait_limit_ns(limit)
                out = torch.empty_like(want)
                call(out)
                status = info.tolist()
                assert status[0] == 0 and status[1] in ((sgdb.SGDB_ERR_TIMEOUT,) if limit == 0 else (sgdb.SGDB_OK, sgdb.SGDB_ERR_TIMEOUT))
                assert status[1] != sgdb.SGDB_OK or torch.equal(out, want)
                sgdb.sgdb_set_wait_limit_ns(-1)
                info.zero_()
                out.fill_(5.0)
                call(out)
                assert info.tolist() == [0, 0] and torch.equal(out, want)
    finally:
        sgdb.sgdb_set_wait_limit_ns(-1)
