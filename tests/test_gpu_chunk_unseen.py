"""Chunks over pages whose rows are not all seen, or not all live: what rows hold that a token does not see does not matter to it, wherever
in a stage of rows they lie.  Against the plain 64-bit form."""
import math
import sys

import pytest
import torch

from paged_ref import assert_within, gather, pages_of
from prompt_ref import CHUNK_CHOICES, attention_rows, causal
from paper_2412_08521_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = B.EMS_BF16, B.EMS_F32


def _log(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _case(n, lens, hq, hkv, d, mode, bad, dead=(), by="positions", ps=16, holds=(math.nan, math.inf), heads=None, seed=0):
    """bad(m): the rows of a sequence of m that are not finite (`holds`: what their keys and values are); dead(m): rows that are
    masked, or (by = "table") whose pages are outside the pool.  Tokens that see no bad row are compared with the
    64-bit form; those that see one are not finite."""
    dt = torch.float32 if mode == F32 else torch.bfloat16
    gen = torch.Generator().manual_seed(seed)
    b, g = len(lens), hq // hkv
    columns, pool = max(-(-m // ps) for m in lens), sum(-(-m // ps) for m in lens) + 3
    table = pages_of(lens, ps, pool, columns, gen)
    kp, vp = (torch.randn((pool, hkv, ps, d), generator=gen).to(dt) for _ in range(2))
    pos = torch.zeros((pool, hkv, ps), dtype=torch.int32) if by == "positions" else None
    lives = []
    for i, m in enumerate(lens):
        live = torch.ones(m, dtype=torch.bool)
        live[[t for t in (dead(m) if dead else ()) if 0 <= t < m]] = False
        for t in bad(m):
            if holds[0] is not None:
                kp[table[i, t // ps], :, t % ps] = holds[0]
            if holds[1] is not None:
                vp[table[i, t // ps], :, t % ps] = holds[1]
        for t in (~live).nonzero()[:, 0].tolist():
            if pos is not None:
                pos[table[i, t // ps], :, t % ps] = -1 - t
        lives.append(live)
    there = table.clone()
    if by == "table":
        for i, live in enumerate(lives):
            for c in range(-(-len(live) // ps)):
                page = live[c * ps:(c + 1) * ps]
                assert page.all() or not page.any()
                if not page.any():
                    there[i, c] = pool if c % 2 else -3
    q = torch.randn((b, hq, n, d), generator=gen).to(dt)
    p = B.PagedParams(b, hq, hkv, d, ps, pool, columns, dtype=mode)
    cache = B.PagedCache(p, kp.cuda(), vp.cuda(), there.cuda(), positions=None if pos is None else pos.cuda())
    o, z = B.ems_paged_chunk_attention(p, cache, torch.tensor(lens, dtype=torch.int32).cuda(), q.cuda(), want_lse=True)
    torch.cuda.synchronize()
    o, z = o.cpu(), z.cpu()
    for i, m in enumerate(lens):
        odd = torch.zeros(m, dtype=torch.bool)
        odd[list(bad(m))] = True
        assert not (odd & ~lives[i]).any()
        for h in heads or range(hq):
            seen = causal(n, m) & lives[i][None]
            fine = ~(seen & odd).any(1)
            ref, zr, bound, zb, _ = attention_rows(q[i, h], gather(kp, table[i], h // g, m), gather(vp, table[i], h // g, m), seen & ~odd,
                                                   d ** -0.5, dt)
            assert_within(o[i, h][fine], ref[fine], bound[fine], f"sequence {i}, head {h}")
            assert_within(z[i, h][fine], zr[fine], zb[fine], f"lse of sequence {i}, head {h}")
            assert not o[i, h][~fine].isfinite().any(), f"sequence {i}, head {h}"


HOLDS = [(math.nan, math.inf), (None, math.nan), (math.nan, None)]


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("by", ["positions", "table"])
@pytest.mark.parametrize("holds", HOLDS)
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (4, 1, 128), (2, 2, 64), (8, 2, 128)])
def test_rows_of_a_stage_whose_first_half_is_dead(hq, hkv, d, holds, by, mode):
    """Of 64 rows the first 50 are dead, and the first live one is seen by the later tokens only: the others' own rows are among the dead."""
    _log("half a stage dead", hq, hkv, d, holds, by, mode)
    _case(40, [80], hq, hkv, d, mode, lambda m: [50], lambda m: range(50), by, ps=10, holds=holds)
    _case(100, [180, 246], hq, hkv, d, mode, lambda m: [m - 180 + 114], lambda m: range(m - 180 + 60, m - 180 + 114), by, ps=6, holds=holds)


@pytest.mark.parametrize("f32,d,b,hq,hkv,n,m,choice", CHUNK_CHOICES)
def test_dead_halves_by_every_choice_of_blocks(f32, d, b, hq, hkv, n, m, choice):
    """The same at each stage that a chunk's tokens end in, for each choice of blocks; sequences that are shorter by some rows move the
    tokens against the stages."""
    _log("dead halves", f32, d, b, hq, hkv, n, m, choice)
    lens = [m - 7 * i if m - 7 * i >= n else m for i in range(b)]
    last = lambda x, at: max(s + at for s in range(0, x, 64) if s + at < x)  # noqa: E731
    for at in (40, 60):
        if all(at < x for x in lens):
            _case(n, lens, hq, hkv, d, F32 if f32 else BF16, lambda x: [last(x, at)],
                  lambda x: [s + t for s in range(0, x, 64) if s + 64 > x - n for t in range(at)], heads=sorted({0, hq // 2, hq - 1}))


# ---- the newest rows are not finite: tokens before them are as they were

def _last(count):
    return lambda m: list(range(m - count, m))


def _some(count, share):
    """Rows apart from the last `count`, `share` of them."""
    def rows(m):
        gen = torch.Generator().manual_seed(m)
        return (torch.rand(m - count, generator=gen) < share).nonzero()[:, 0].tolist()
    return rows


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("share", [None, 0.0, 0.3, 0.9])               # of masked rows; None: a cache without positions
@pytest.mark.parametrize("holds", HOLDS + [(None, -math.inf), (math.inf, None)])
@pytest.mark.parametrize("hq,hkv,d,n,lens", [
    (8, 2, 128, 4, [4, 70, 33, 5]), (4, 1, 64, 8, [64, 700]), (1, 1, 128, 32, [32, 33, 3000]), (2, 1, 64, 16, [16, 47, 128]),
    (4, 4, 64, 5, [2001, 129, 17]), (20, 2, 128, 3, [131, 3]), (4, 2, 128, 2, [6000]), (3, 1, 64, 10, [48] * 70)])
def test_few_columns_whose_newest_rows_are_not_finite(hq, hkv, d, n, lens, holds, share, mode):
    _log("few columns", hq, hkv, d, n, lens, holds, share, mode)
    count = min(3, n - 1)
    _case(n, lens, hq, hkv, d, mode, _last(count), _some(count, share) if share else (), "table" if share is None else "positions", holds=holds)


@pytest.mark.parametrize("share", [None, 0.0, 0.3, 0.9])
@pytest.mark.parametrize("holds", HOLDS)
@pytest.mark.parametrize("f32,d,b,hq,hkv,n,m,choice", CHUNK_CHOICES)
def test_newest_rows_by_every_choice_of_blocks(f32, d, b, hq, hkv, n, m, choice, holds, share):
    _log("newest rows", f32, d, b, hq, hkv, n, m, choice, holds, share)
    lens = [max(n, m - 150 * i) for i in range(b)]
    _case(n, lens, hq, hkv, d, F32 if f32 else BF16, _last(3), _some(3, share) if share else (), "table" if share is None else "positions",
          holds=holds, heads=sorted({0, hq // 2, hq - 1}))
