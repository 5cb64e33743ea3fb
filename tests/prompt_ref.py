"""Plain 64-bit form of the attention of many queries, each over rows of its own, on the CPU, with bounds on what 32-bit arithmetic, weights
of 16 bits and one rounding to the tensors' type may leave between a kernel and it."""
import math

import torch

from paged_ref import F32, half_step


def attention_rows(q, k, v, seen, scale, dtype):
    """q [N, D], k, v [M, D], seen [N, M] -> out, lse, bound of out, bound of lse, variance of out's rounding errors.

    A logit is off by at most D half steps of the sum of its products' moduli and a few of its own size; a weight by that,
    twice (its own and the reference's), and the additions that the sums take.  In 16-bit products a weight is rounded to
    bf16 once (the sum that divides is of the weights before), half a step of it at most; the output is rounded once.  A
    rounding of half a step h at most has a variance of h^2 / 3 at most, and the weights' are independent."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    used = seen.any(0)                                     # rows that nobody sees may hold anything
    k = torch.where(used[:, None], k, 0.0)
    v = torch.where(used[:, None], v, 0.0)
    if k.shape[0] == 0:
        zero = torch.zeros(n, d, dtype=torch.float64)
        return zero, torch.full((n,), -math.inf, dtype=torch.float64), zero, torch.zeros(n, dtype=torch.float64), zero
    x = q @ k.T * scale
    size = torch.where(seen, (q.abs() @ k.abs().T * scale), 0.0).amax(1)
    top = torch.where(seen, x.abs(), 0.0).amax(1)
    x = torch.where(seen, x, -math.inf)
    z = torch.logsumexp(x, 1)
    p = torch.where(seen, (x - torch.where(z > -math.inf, z, 0.0)[:, None]).exp(), 0.0)
    out = p @ v
    logit = (size * (d + 4) + 4 * top + 4) * F32
    count = seen.sum(1).double()
    rounded = half_step(torch.bfloat16) if dtype == torch.bfloat16 else 0.0
    rel = 2 * logit + 2 * (count + 8) * F32 + rounded
    bound = rel[:, None] * (p @ v.abs()) + out.abs() * half_step(dtype) * (1 + 2.0 ** -6)
    var = (rounded ** 2 * (p ** 2 @ v ** 2) + half_step(dtype) ** 2 * out ** 2) / 3
    lse_bound = torch.where(z > -math.inf, logit + (count + 8) * F32 + 4 * F32 * z.abs(), 0.0)
    return out, z, bound + torch.finfo(dtype).tiny, lse_bound, var


def causal(n, m):
    """Query i of n sees rows t <= i + m - n of m."""
    return torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n)


def plan(batch, q_heads, kv_heads, head_dim, q_rows, k_rows, packed=False, paged=False, f32=False):
    """(waves of a block's rows, blocks that share a tile's rows of keys and values) that a call takes: the launcher's own choice."""
    import ctypes as C

    from paper_2412_08521_amd import binding as B

    class Plan(C.Structure):
        _fields_ = [("waves", C.c_int), ("splits", C.c_int), ("tiles", C.c_longlong)]
    f = getattr(B.lib(), "_ZN3ems11plan_promptExxxiiixbb")
    f.restype = Plan
    f.argtypes = [C.c_longlong] * 3 + [C.c_int] * 3 + [C.c_longlong, C.c_bool, C.c_bool]
    g = q_heads // kv_heads
    p = f(batch, q_rows * g, q_rows * g if packed else batch * q_rows * g, kv_heads, g, head_dim, max(k_rows, 1), paged, f32)
    return p.waves, p.splits


# Calls that take each choice of plan(): float32, head size, sequences, q-heads, kv-heads, queries and rows of a sequence, the choice.
CHOICES = [
    (False, 64, 1, 4, 4, 300, 300, (1, 1)), (False, 64, 1, 32, 8, 40, 3000, (1, 4)), (False, 64, 1, 4, 4, 40, 3000, (1, 8)),
    (False, 64, 1, 4, 4, 33, 33, (2, 1)), (False, 64, 4, 16, 8, 520, 1000, (4, 1)), (False, 64, 8, 32, 8, 200, 2000, (8, 1)),
    (False, 128, 1, 4, 4, 300, 300, (1, 1)), (False, 128, 1, 4, 4, 200, 2000, (1, 4)), (False, 128, 1, 4, 4, 40, 3000, (1, 8)),
    (False, 128, 1, 4, 4, 33, 33, (2, 1)), (False, 128, 4, 16, 8, 520, 1000, (4, 1)), (False, 128, 1, 4, 4, 4097, 4097, (4, 2)),
    (False, 128, 8, 32, 8, 200, 2000, (8, 1)),
    (True, 64, 4, 16, 8, 520, 1000, (2, 1)), (True, 128, 1, 4, 4, 200, 2000, (2, 8)),
]
CHUNK_CHOICES = [
    (False, 64, 1, 4, 4, 300, 304, (1, 1)), (False, 64, 1, 4, 4, 40, 3008, (1, 8)), (False, 64, 1, 4, 4, 33, 48, (2, 1)),
    (False, 64, 8, 32, 8, 40, 3008, (2, 2)), (False, 64, 4, 16, 8, 520, 1008, (4, 1)), (False, 64, 8, 32, 8, 200, 2000, (8, 1)),
    (False, 128, 1, 4, 4, 300, 304, (1, 1)), (False, 128, 2, 8, 8, 200, 2000, (1, 2)), (False, 128, 1, 4, 4, 200, 2000, (1, 4)),
    (False, 128, 1, 4, 4, 40, 3008, (1, 8)), (False, 128, 1, 4, 4, 33, 48, (2, 1)), (False, 128, 1, 32, 8, 40, 3008, (2, 8)),
    (False, 128, 8, 32, 8, 100, 112, (4, 1)), (False, 128, 4, 16, 8, 200, 2000, (4, 2)), (False, 128, 4, 16, 8, 40, 3008, (4, 8)),
    (False, 128, 8, 32, 8, 500, 512, (8, 1)),
    (True, 64, 4, 16, 8, 520, 1008, (2, 1)), (True, 128, 1, 4, 4, 200, 2000, (2, 8)),
]
