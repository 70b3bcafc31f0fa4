"""Numbers in 8 bits with a power of two for each block of 128, in elementary torch operations on any device: what the kernels'
results are compared with.  Written from the header's definition."""
import torch

FORMATS = [torch.float8_e4m3fn, torch.float8_e5m2]
LOWEST = -110


def exponents(x, largest):
    """Of the last dimension: the smallest e >= LOWEST with max|finite x| <= largest 2^e, 0 where there is none but zeros."""
    top = torch.where(torch.isfinite(x), x.double().abs(), 0.0).amax(-1)
    e = torch.ceil(torch.log2(torch.where(top > 0, top / largest, 1.0)))
    e = torch.where(torch.exp2(e) * largest < top, e + 1, e)  # the logarithm may be off by its last bit
    e = torch.where(torch.exp2(e - 1) * largest >= top, e - 1, e)
    return torch.where(top > 0, e, 0.0).clamp(min=LOWEST)


def rounded(x, e, fmt):
    v = x.double() * torch.exp2(-e)
    v = torch.where(torch.isfinite(x), v, torch.nan)
    return v.float().to(fmt)  # exact to float32 but for numbers far below the format's smallest


def padded(x, dim):
    more = -x.shape[dim] % 128
    shape = list(x.shape)
    shape[dim] = more
    return torch.cat([x, x.new_zeros(shape)], dim) if more else x


def quantized(x, fmt):
    """x [..., width] -> q of the same shape, e [..., blocks] as float64."""
    b = padded(x, -1).unflatten(-1, (-1, 128))
    e = exponents(b, torch.finfo(fmt).max)
    return rounded(b, e[..., None], fmt).flatten(-2)[..., : x.shape[-1]], e


def quantized_matrices(w, fmt):
    """w [batch, rows, cols] -> q, e [batch, row blocks, column blocks]."""
    b = padded(padded(w, -1), -2).unflatten(-1, (-1, 128)).unflatten(-3, (-1, 128)).transpose(-3, -2)
    e = exponents(b.flatten(-2), torch.finfo(fmt).max)
    q = rounded(b, e[..., None, None], fmt).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    return q[..., : w.shape[-2], : w.shape[-1]], e


def scales(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def wide(q, scale):
    """The values in 64 bits; scale: float8_e8m0fnu, or the numbers in 64 bits."""
    return q.to(torch.float64) * scale.to(torch.float64).repeat_interleave(128, -1)[..., : q.shape[-1]]


def wide_matrices(q, scale):
    return wide(q, scale.to(torch.float64).repeat_interleave(128, -2)[..., : q.shape[-2], :])


def same8(a, b):
    """Equal values, NaN alike."""
    a, b = a.float(), b.float()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())
