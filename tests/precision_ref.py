"""How precise the attention of one new token has to be: inputs whose outputs show the weights' last digits, and the
standard deviation that rounding in 32 bits leaves.  On the CPU, in 64 bits."""
import math

import torch

U = 2.0 ** -24                       # half a step of float32, relative to the value


# ---- values that cancel what 16 or 17 bits of a weight hold

def cancelling(group, d, seed, dtype):
    """-> (q [group, d], k [3, d], v [3, d], scale).  Rows 0 and 1 have logit 0, row 2 has logit -x_j for q-head j, so its
    weight is p_j = exp(-x_j) times theirs, in (1/8, 1).  Column j of the values is (hi, mid, -1) with hi + mid the two-piece
    bf16 form of p_j: out[j, j] = (hi + mid - p_j) / (2 + p_j), up to 2^-17 of p_j, which is what a weight of two bf16
    pieces (or of fewer digits) makes 0 or worse.  (q-heads past d have no column of their own.)"""
    gen = torch.Generator().manual_seed(seed)
    q = torch.zeros(group, d)
    q[:, 0] = (0.05 + 2.0 * torch.rand(group, generator=gen)).bfloat16().float()
    k = torch.zeros(3, d)
    k[2, 0] = -1.0
    p = (-q[:, 0].double()).exp()
    v = torch.zeros(3, d)
    n = min(group, d)
    hi = p.float().bfloat16().double()
    v[0, :n] = hi[:n].float()
    v[1, :n] = (p - hi)[:n].float().bfloat16().float()
    v[2, :n] = -1.0
    return q.to(dtype), k.to(dtype), v.to(dtype), 1.0


def cancelling_bound(q, dtype):
    """-> (out[j, j], bound), [group].  The logit is one product: itself exact, times the scale and log2(e), whose 32-bit
    value is half a step off: 3 half steps of x.  The exponential: 2 steps of p.  Three products, up to three pieces each,
    added to a sum of at most 2 p: 9 additions of a whole step at most of it; the division and the weights' sum 4 more."""
    x = q[:, 0].double()
    p = (-x).exp()
    hi = p.float().bfloat16().double()
    mid = (p - hi).float().bfloat16().double()
    out = (hi + mid - p) / (2 + p)
    each = p * (3 * x + 4) * U + 2 * p * 9 * 2 * U
    return out, each / (2 + p) + out.abs() * (4 * U + torch.finfo(dtype).eps / 2 * (1 + 2.0 ** -6))


# ---- the rms of the error

def rms_parts(q, k, v, live, scale):
    """q [G, D], k, v [L, D], live [L] -> (out, variance of its error) in 64 bits.  Roundings are taken as independent and
    uniform (variance U^2 / 3 of the rounded value's square): D additions to a logit, its scaling and the exponential (4 more
    of the logit, 2 of the probability), and the L additions to the sum of weights and of weighted values, in order."""
    q, k, v = q.double(), k.double()[live], v.double()[live]
    if len(k) == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    x = q @ k.T * scale
    z = torch.logsumexp(x, 1, keepdim=True)
    w = (x - z).exp()
    out = w @ v
    rel = 4 * x.square() + 2
    for g in range(len(q)):                                  # partial sums of the products, a q-head at a time
        rel[g] += (q[g] * k * scale).cumsum(1).square().sum(1)
    ww = w.square() * rel
    # weight errors act through v_t - out
    var = ww @ v.square() - 2 * out * (ww @ v) + out.square() * ww.sum(1, keepdim=True)
    for g in range(len(q)):
        var[g] += (w[g][:, None] * v).cumsum(0).square().sum(0)
        var[g] += out[g].square() * w[g].cumsum(0).square().sum()
    return out, var.clamp(min=0) * U * U / 3


class Rms:
    """Errors of a whole case against what their variances allow."""

    def __init__(self, dtype):
        self.dtype, self.n, self.off, self.var, self.own = dtype, 0, 0.0, 0.0, 0.0

    def add(self, got, out, var):
        assert got.isfinite().all()
        self.n += out.numel()
        self.off += float((got.double() - out).square().sum())
        self.own += float((out.to(self.dtype).double() - out).square().sum())       # the one rounding to the output's type
        self.var += float(var.sum())

    def ratio(self):
        """The rms error beyond the output's own rounding, in standard deviations; must stay under 3 (twice the deviation
        that the model gives, for sums in another order and instructions that cut instead of rounding, plus what the own
        rounding of an output that is off already may add)."""
        beyond = max(0.0, self.off - self.own * (1 + self.slack()))
        return math.sqrt(beyond / self.var) if self.var else (0.0 if beyond == 0 else math.inf)

    def slack(self):
        """Rounding off + e instead of off adds a term of 2 E[r e], which is 0 on average: r is uniform in half a step and an e
        that turns it into the next step does so from either side.  Its deviation over n values is 2 sqrt(own var) / sqrt(n)
        of the sum; four of them, relative to own."""
        return 8 * math.sqrt(self.var / self.own / self.n) if self.own else 0.0


def plain(q, k, v, live, scale, dtype, weights):
    """The attention in 32 bits with `weights` applied to the probabilities of the numerator, one rounding at the end."""
    q, k, v = q.float(), k.float()[live], v.float()[live]
    x = q @ k.T * scale
    p = (x - x.amax(1, keepdim=True)).exp()
    return (weights(p) @ v / p.sum(1, keepdim=True)).to(dtype)


def pieces(n):
    def split(p):
        total = torch.zeros_like(p, dtype=torch.float64)
        rest = p.clone()
        for _ in range(n):
            one = rest.bfloat16().float()
            total += one
            rest = rest - one
        return total.float()
    return split
