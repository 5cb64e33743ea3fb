"""Attention of one new token where blocks take several units and cross sequences, and where a wave packs live rows by the
hundred (tests/test_attention_split_host.py holds that these shapes do)."""
import math
import sys

import pytest
import torch

from attention_checks import check
from paged_ref import assert_within, attention, gather
from paper_2412_08521_amd import binding as B
from test_gpu_decode_attention import _check, _made_up, _token
from test_gpu_paged import _attend_case

pytestmark = pytest.mark.gpu

BF16, F32 = B.EMS_BF16, B.EMS_F32
MODES = [BF16, F32]

# b, hq, hkv, d, page size, lengths, columns
SHARED = {
    "ragged": (12, 64, 32, 64, 16, [0, 777, 0, 2000, 1, 0, 0, 128, 1290, 129, 1999, 0], 380),
    "even": (7, 32, 32, 64, 16, [512, 1024, 512, 2048, 1024, 512, 512], 380),          # 48 units for 24 workers
    "many": (150, 16, 8, 64, 32, [(37 * i * i) % 900 for i in range(75)] + [0, 2900, 0] + [(53 * i) % 500 for i in range(72)], 140),
    "tiles": (9, 320, 16, 64, 16, [0, 3000, 5, 1500, 260, 0, 2000, 999, 1100], 400),   # 20 q-heads a kv-head
    "wide": (8, 64, 32, 128, 24, [1700, 0, 300, 1201, 64, 2040, 0, 513], 200),
    "caches": (2, 32, 32, 64, 16, [2100, 2283], 145),         # rows that stay in the caches
}

COMPACT = [
    # b, hq, hkv, d, budget, window, ratio
    (3, 64, 32, 64, 1450, 32, 0.5),
    (4, 32, 32, 128, 1100, 16, 0.25),
    (3, 640, 32, 64, 1400, 16, 0.5),
]

_WHOLE = [1500, 1024, 3, 0, 64, 1333, 128, 31, 1290]
RINGS = {
    "whole 64": ((9, 64, 64, 64, 16, _WHOLE, 110), BF16),
    "whole 64 float32": ((9, 64, 64, 64, 16, _WHOLE, 110), F32),
    "whole 128": ((9, 128, 64, 128, 16, _WHOLE, 110), BF16),
    "whole 128 float32": ((9, 64, 64, 128, 16, [1000, 1024, 3, 0, 64, 1023, 128, 31, 900], 64), F32),
    "shared 64": ((6, 96, 48, 64, 16, [3000, 5, 4200, 0, 2900, 2500], 380), BF16),
    "shared 128": ((6, 48, 48, 128, 32, [3000, 5, 4200, 0, 2900, 2500], 180), BF16),
    "shared 128 float32": ((5, 48, 48, 128, 16, [3000, 5, 4200, 0, 2900], 380), F32),
    "shared tiles": ((5, 960, 48, 64, 16, [3100, 5, 4200, 0, 5900], 380), BF16),
    "shared tiles float32": ((5, 960, 48, 64, 16, [3100, 5, 4200, 0, 5900], 380), F32),
}


def _log(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def paged_params(shape, mode, pool):
    b, hq, hkv, d, ps, _, columns = shape
    return B.PagedParams(b, hq, hkv, d, ps, pool, columns, dtype=mode)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("masked", [None, 0.3])
@pytest.mark.parametrize("name", sorted(SHARED))
def test_workers_of_several_units(name, masked, mode):
    _log("shared", name, masked, mode)
    shape = SHARED[name]
    p, cache, lens, q, out = _attend_case(*shape[:6], mode, masked=masked, columns=shape[6], seed=len(name))
    lse = B.ems_paged_attention(p, cache, lens, q, want_lse=True)[1]
    check(p, cache, lens, q, out, lse)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shape", COMPACT)
def test_compact_workers_of_several_units(shape, mode):
    _log("compact", shape, mode)
    p, st, gen = _made_up(*shape, mode, seed=shape[4])
    q, k, v = _token(p, gen)
    out, lse = B.ems_decode_attention(p, st, q.cuda(), k.cuda(), v.cuda(), want_lse=True)
    _check(p, st, q, k, v, out, lse)


def _ring_case(name, seed):
    """Inputs of a packed attention with all rows live, made on the device: heads of normal keys with a heavy direction."""
    shape, mode = RINGS[name]
    b, hq, hkv, d, ps, lens, columns = shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    counts = [-(-n // ps) for n in lens]
    pool = sum(counts) + 1
    p = paged_params(shape, mode, pool)
    randn = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    u = torch.nn.functional.normalize(randn(hkv, 1, d), dim=-1)
    heavy = torch.empty((pool, hkv, ps, 1), device="cuda").exponential_(1.0, generator=gen)
    k = (randn(pool, hkv, ps, d) + 0.25 * math.sqrt(d) * heavy * u).to(p.torch_dtype)
    v = randn(pool, hkv, ps, d).to(p.torch_dtype)
    q = (randn(b, hkv, hq // hkv, d) + 4.0 * u).view(b, hq, d).to(p.torch_dtype)
    order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((b, columns), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n
    pos = torch.zeros((pool, hkv, ps), dtype=torch.int32, device="cuda")
    return p, B.PagedCache(p, k, v, table, positions=pos), torch.tensor(lens, dtype=torch.int32, device="cuda"), q, gen


def _mask(p, cache, lens, live):
    """live(sequence, rows) -> [kv_heads, rows] bool; masked rows, and those of nobody, hold NaN and infinities."""
    pos = torch.full_like(cache.positions, -1)
    for i, n in enumerate(lens.tolist()):
        rows = torch.arange(n, device="cuda")
        page, at = cache.page_table[i].long()[rows // p.page_size], rows % p.page_size
        pos[page, :, at] = torch.where(live(i, n).T, 7, -1).to(torch.int32)
    cache.positions.copy_(pos)
    for x, bad in ((cache.k_pages, math.nan), (cache.v_pages, math.inf)):
        x[pos < 0] = bad


def _clustered(p, gen):
    """Runs of 256 rows (a wave's look at two turns) that are live, dead or hold one live row."""
    def live(i, n):
        runs = torch.randint(0, 3, (p.kv_heads, n // 256 + 1), device="cuda", generator=gen).repeat_interleave(256, 1)[:, :n]
        one = torch.randint(0, 256, (p.kv_heads, 1), device="cuda", generator=gen)
        return (runs == 0) | ((runs == 1) & (torch.arange(n, device="cuda") % 256 == one))
    return live


@pytest.mark.parametrize("share", [0.0, 0.02, 0.6, 0.97, "runs"])
@pytest.mark.parametrize("name", sorted(RINGS))
def test_rings_that_wrap(name, share):
    _log("ring", name, share)
    p, cache, lens, q, gen = _ring_case(name, len(name))
    if share == "runs":
        _mask(p, cache, lens, _clustered(p, gen))
    else:
        _mask(p, cache, lens, lambda i, n: torch.rand((p.kv_heads, n), device="cuda", generator=gen) >= share)
    out, lse = B.ems_paged_attention(p, cache, lens, q, want_lse=True)
    assert torch.equal(out, B.ems_paged_attention(p, cache, lens, q))
    # all of a sequence's heads are one kernel's work: a few of them for the 64-bit form
    keep = sorted({0, 1, p.kv_heads // 2, p.kv_heads - 1})
    g = p.q_heads // p.kv_heads
    heads = torch.tensor([h * g + j for h in keep for j in range(g)], device="cuda")
    few = B.PagedParams(p.batch, len(keep) * g, len(keep), p.head_dim, p.page_size, p.num_pages, p.max_pages, dtype=p.dtype)
    part = B.PagedCache(few, *(x[:, keep].contiguous() for x in (cache.k_pages, cache.v_pages)), cache.page_table,
                        positions=cache.positions[:, keep].contiguous())
    check(few, part, lens, q[:, heads], out[:, heads], lse[:, heads])


# ---- live rows that are not finite

@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("group", [4, 20])
@pytest.mark.parametrize("rows,columns", [(200, 13), (900, 70), (900, 24000)])          # whole, shared, past the caches (packed)
def test_live_rows_that_are_not_finite(rows, columns, group, masked, mode):
    _log("not finite", rows, columns, group, masked, mode)
    b, hkv, d, ps = 2, 3, 64, 16
    gen = torch.Generator().manual_seed(rows + group)
    n_pages = -(-rows // ps)
    p = B.PagedParams(b, hkv * group, hkv, d, ps, b * n_pages, columns, dtype=mode)
    table = torch.full((b, columns), -1, dtype=torch.int32)
    table[:, :n_pages] = torch.arange(b * n_pages).view(b, n_pages)
    k, v = (torch.randn((b * n_pages, hkv, ps, d), generator=gen).to(p.torch_dtype) for _ in range(2))
    q = torch.randn((b, hkv * group, d), generator=gen)
    q[..., 0] = q[..., 0].abs() + 0.5
    q = q.to(p.torch_dtype)
    pos = torch.randint(-1, 2, k.shape[:3], generator=gen, dtype=torch.int32) if masked else None
    spots = [5, rows // 2 + 3, rows - 1]                     # of sequence 0
    at = lambda t: (t // ps, t % ps)  # noqa: E731
    if masked:
        for t in spots:
            pos[at(t)[0], :, at(t)[1]] = 3
    lens = torch.full((b,), rows, dtype=torch.int32)

    def run(k, v):
        cache = B.PagedCache(p, k.cuda(), v.cuda(), table.cuda(), positions=pos.cuda() if masked else None)
        return [x.cpu() for x in B.ems_paged_attention(p, cache, lens.cuda(), q.cuda(), want_lse=True)]
    out0, lse0 = run(k, v)
    assert out0.isfinite().all() and lse0.isfinite().all()
    for t in spots:
        page, row = at(t)
        # a value: its column of its sequence-head, nothing else
        for bad in (math.inf, -math.inf, math.nan):
            w = v.clone()
            w[page, 1, row, 7] = bad
            out, lse = run(k, w)
            off = ~out.isfinite()
            assert off[0, group:2 * group, 7].all() and off.sum() == group
            assert torch.equal(out[~off], out0[~off]) and torch.equal(lse, lse0)
        # a key of NaN, or an infinite logit: its sequence-head, nothing else
        for bad in (math.nan, math.inf):
            x = k.clone()
            x[page, 1, row, 0] = bad
            out, lse = run(x, v)
            off = ~out.isfinite()
            assert off[0, group:2 * group].all() and off.sum() == group * d and not lse[0, group:2 * group].isfinite().any()
            assert torch.equal(out[~off], out0[~off])
        # a logit of -inf weighs nothing
        x = k.clone()
        x[page, 1, row, 0] = -math.inf
        out, lse = run(x, v)
        live = gather(pos, table[0], 1, rows) >= 0 if masked else torch.ones(rows, dtype=torch.bool)
        live[t] = False
        heads = slice(group, 2 * group)
        ref = attention(q[0, heads], gather(k, table[0], 1, rows), gather(v, table[0], 1, rows), live, d ** -0.5, p.torch_dtype)
        assert_within(out[0, heads], ref[0], ref[2], f"row {t} of -inf")
        assert_within(lse[0, heads], ref[1], ref[3], f"row {t} of -inf, lse")


# ---- pages of several sequences

@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("masked", [None, 0.4])
@pytest.mark.parametrize("columns", [None, 20000])
def test_sequences_that_share_pages(columns, masked, mode):
    """A common start on the same pages gives what a copy of it for every sequence gives, and 64 bits say."""
    _log("pages shared", columns, masked, mode)
    p, cache, _, q, _ = _attend_case(3, 8, 2, 64, 16, [1500, 900, 40], mode, masked=masked, columns=columns, poison=False, seed=5)
    table = cache.page_table.clone()
    table[1, :50] = table[0, :50]
    table[2, :94] = table[0, :94]
    table[2, 50:94] = table[0, 50:94].flip(0)                # in another order, the same pages
    table[1, 50:] = -1
    lens = torch.tensor([1500, 800, 1500], dtype=torch.int32).cuda()
    shared = B.PagedCache(p, cache.k_pages, cache.v_pages, table, positions=cache.positions)
    out, lse = B.ems_paged_attention(p, shared, lens, q, want_lse=True)
    check(p, shared, lens, q, out, lse)
    pages = torch.cat([table[i, :-(-n // 16)] for i, n in enumerate(lens.tolist())]).long()
    own = torch.full_like(table, -1)
    at = 0
    for i, n in enumerate(lens.tolist()):
        m = -(-n // 16)
        own[i, :m] = torch.arange(at, at + m)
        at += m
    p2 = B.PagedParams(3, 8, 2, 64, 16, at, p.max_pages, dtype=mode)
    copy = B.PagedCache(p2, cache.k_pages[pages], cache.v_pages[pages], own,
                        positions=cache.positions[pages] if masked is not None else None)
    assert all(torch.equal(x, y) for x, y in zip((out, lse), B.ems_paged_attention(p2, copy, lens, q, want_lse=True)))
