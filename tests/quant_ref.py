"""Plain form of rows in 8 bits: e4m3 numbers and a power of two a row."""
import torch


def top_of(x):
    """The largest modulus of the finite elements of rows [.., D]."""
    return torch.where(x.isfinite(), x, 0.0).abs().amax(-1)


def exponent(top):
    """s: the smallest, not below -126, with top <= 448 2^s."""
    mant, exp = torch.frexp(top.double())                  # top = mant 2^exp, mant in [1/2, 1); 448 = 7/8 2^9
    s = exp - 9 + (mant > 0.875).to(exp.dtype)
    return torch.where(top > 0, s, -126).clamp(min=-126).to(torch.int32)


def codes(x, s):
    """Rows in 64 bits and their exponents -> e4m3 numbers, by hand: steps of 2^-3 of the leading power of two, from 2^-6 down
    2^-9."""
    y = x.double() * torch.exp2(-s.double())[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))) / 8
    near = torch.round(y / step) * step                    # ties to even
    return torch.where(x.isfinite(), near, torch.nan)


def values(pages, scale):
    """What pages [.., D] float8_e4m3fn and their bytes stand for, in 64 bits."""
    return pages.float().double() * torch.exp2(scale.double() - 127)[..., None]
