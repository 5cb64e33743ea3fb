"""Plain 64-bit forms of the paged append and of the attention of one new token, on the CPU, with bounds on what 32-bit
arithmetic and one rounding to the tensors' type may leave between a kernel and them."""
import math

import torch

F32 = 2.0 ** -24                     # half a step of float32, relative to the value


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rotated(x, pos, inv_freq, interleaved):
    """x [..., N, D], pos [..., N] -> (rotated, bound of the 32-bit part of its error).  Cosine, sine (4 half steps each:
    the cut angle, the function), two products and a sum: 8 half steps of |x1| + |x2| are more than all of them."""
    x = x.double().clone()
    slack = torch.zeros_like(x)
    if inv_freq is None:
        return x, slack
    half = inv_freq.numel()
    e = torch.arange(half)
    one, two = (2 * e, 2 * e + 1) if interleaved else (e, e + half)
    a = pos.double()[..., None] * inv_freq.double()
    c, s = a.cos(), a.sin()
    u, w = x[..., one], x[..., two]
    x[..., one], x[..., two] = u * c - w * s, w * c + u * s
    slack[..., one] = slack[..., two] = 8 * F32 * (u.abs() + w.abs())
    return x, slack


def attention(q, k, v, live, scale, dtype):
    """q [G, D], k, v [L, D], live [L] -> (out, lse, bound of out, bound of lse).

    A logit is off by at most D half steps of the sum of its products' moduli and a few of its own size (scaled logit,
    exponent); a probability by that, twice (its own and the largest's), 2^-17 where it goes into 16-bit products as two
    pieces, and the n additions that the sums take."""
    q, k, v = q.double(), k.double()[live], v.double()[live]
    g, d = q.shape
    if len(k) == 0:
        zero = torch.zeros(g, d, dtype=torch.float64)
        return zero, torch.full((g,), -math.inf, dtype=torch.float64), zero, torch.zeros(g, dtype=torch.float64)
    x = q @ k.T * scale
    z = torch.logsumexp(x, 1)
    p = (x - z[:, None]).exp()
    out = p @ v
    logit = ((q.abs() @ k.abs().T * scale).amax(1) * (d + 4) + 4 * x.abs().amax(1) + 4) * F32
    pieces = 2.0 ** -16 if dtype == torch.bfloat16 else 0.0
    rel = 2 * logit + pieces + 2 * (len(k) + 8) * F32
    bound = rel[:, None] * (p @ v.abs()) + out.abs() * half_step(dtype) * (1 + 2.0 ** -6)
    return out, z, bound + torch.finfo(dtype).tiny, logit + (len(k) + 8) * F32 + 4 * F32 * z.abs()


def assert_within(got, ref, bound, what):
    got = got.detach().cpu().double()
    off = (got - ref).abs()
    same = got == ref                              # infinities
    bad = ~(same | (off <= bound))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {(off / bound.clamp(min=1e-300))[bad].max():.3g} bounds"


def pages_of(lens, page_size, pool, columns, gen):
    """A table whose rows name pages in no order; columns behind a sequence's last page hold numbers of no page."""
    order = torch.randperm(pool, generator=gen).to(torch.int32)
    table = torch.full((len(lens), columns), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-n // page_size)
        table[b, :m] = order[at:at + m]
        table[b, m + 1:] = 1 << 30
        at += m
    return table


def gather(pages, table_row, head, n):
    """The first n rows of a sequence's kv-head."""
    ps = pages.shape[2]
    return pages[table_row[:-(-n // ps)].long(), head].flatten(0, 1)[:n]
