"""Checks of a paged attention's outputs from the tensors that the call had, and how a call's work is split."""
import ctypes as C

import torch

from paged_ref import assert_within, attention, gather
from paper_2412_08521_amd import binding as B
from precision_ref import Rms, rms_parts

UNIT = 128                                        # rows that work is counted in


def check(p, cache, lens, q, out, lse, worst=3.0):
    """Every element within its bound, and the rms of the error within `worst` deviations."""
    k_pages, v_pages, table, q, out, lse = (x.cpu() for x in (cache.k_pages, cache.v_pages, cache.page_table, q, out, lse))
    pos = cache.positions.cpu() if cache.positions is not None else torch.zeros(p._pages[:3], dtype=torch.int32)
    scale = p.softmax_scale if p.softmax_scale > 0 else p.head_dim ** -0.5
    rms, g = Rms(p.torch_dtype), p.q_heads // p.kv_heads
    for i, n in enumerate(lens.tolist()):
        for h in range(p.kv_heads):
            heads = slice(h * g, (h + 1) * g)
            k, v, live = (gather(x, table[i], h, n) for x in (k_pages, v_pages, pos >= 0))
            ref = attention(q[i, heads], k, v, live, scale, p.torch_dtype)
            assert_within(out[i, heads], ref[0], ref[2], f"out of {i}, {h} ({n} rows)")
            assert_within(lse[i, heads], ref[1], ref[3], f"lse of {i}, {h} ({n} rows)")
            rms.add(out[i, heads], *rms_parts(q[i, heads], k, v, live, scale))
    assert rms.ratio() < worst, rms.ratio()


def workers(batch, kv_heads, group, max_len, row_bytes):
    """Blocks that share a kv-head's sequences (0: a block per sequence), as the host side decides it."""
    f = getattr(B.lib(), "_ZN3ems14attend_workersEiiixi")
    f.restype, f.argtypes = C.c_int, [C.c_int] * 3 + [C.c_longlong, C.c_int]
    return f(batch, kv_heads, group, max_len, row_bytes)


def stretches(lens, n_workers):
    """What each worker takes: [(sequence, first unit of it, units of it taken, units it has), ...]."""
    units = [-(-n // UNIT) for n in lens]
    total = sum(units)
    per, more = divmod(total, n_workers)
    owner = [(b, u) for b, n in enumerate(units) for u in range(n)]
    taken, at = [], 0
    for w in range(n_workers):
        mine = owner[at:at + per + (w < more)]
        at += len(mine)
        one = []
        for b in sorted({b for b, _ in mine}):
            first = [u for c, u in mine if c == b]
            one.append((b, first[0], len(first), units[b]))
        taken.append(one)
    return taken
