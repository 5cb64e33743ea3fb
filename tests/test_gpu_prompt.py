"""GPU parity of the attention of whole prompts (ems_prompt_attention) and of chunks over pages (ems_paged_chunk_attention) with a
plain 64-bit form."""
import math
import sys

import pytest
import torch

from paged_ref import assert_within, gather, pages_of
from prompt_ref import CHOICES, CHUNK_CHOICES, attention_rows, causal
from paper_2412_08521_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = B.EMS_BF16, B.EMS_F32


def _log(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _dtype(mode):
    return torch.float32 if mode == F32 else torch.bfloat16


def _laid_out(x, layout):
    """x [.., tokens, heads, D] on the device as a view of memory of that layout."""
    if layout == "tokens":
        return x.cuda()
    if layout == "heads":                                   # heads before tokens
        return x.transpose(-3, -2).contiguous().cuda().transpose(-3, -2)
    if layout == "wide":                                    # rows with something between them, 16-byte aligned
        big = torch.full(x.shape[:-1] + (x.shape[-1] + 16,), math.nan, dtype=x.dtype)
        big[..., 8:8 + x.shape[-1]] = x
        return big.cuda()[..., 8:8 + x.shape[-1]]
    assert layout == "odd"                                  # no row aligned to more than an element
    big = torch.full((x.numel() // x.shape[-1] * (x.shape[-1] + 1) + 1,), math.nan, dtype=x.dtype)
    big[1:].view(x.shape[:-1] + (x.shape[-1] + 1,))[..., :-1] = x
    return big.cuda()[1:].view(x.shape[:-1] + (x.shape[-1] + 1,))[..., :-1]


class Rms:
    """The errors of a case together: their mean square at most half as much again as the roundings' variance (tens of thousands
    of elements; in float32 the bound of each element says it all)."""

    def __init__(self):
        self.off, self.var, self.n = 0.0, 0.0, 0

    def add(self, got, ref, var):
        self.off += float((got.cpu().double() - ref).square().sum())
        self.var += float(var.sum())
        self.n += ref.numel()

    def check(self, mode):
        if mode == BF16 and self.n >= 20000:
            assert self.off <= 1.5 * self.var, (self.off / self.var, self.n)


def _prompt_case(lens, hq, hkv, d, mode, before=None, packed=False, layout="tokens", out_layout="tokens", spare=(0, 0), seed=0,
                 scale=0.0, poison=False, hot=1.0, heads=None):
    """lens: queries of every sequence; before: rows of keys and values before them (may be negative: fewer rows than queries)."""
    dt = _dtype(mode)
    gen = torch.Generator().manual_seed(seed)
    rows = [max(0, n + m) for n, m in zip(lens, before or [0] * len(lens))]
    b = len(lens)
    n, m = (sum(lens) + sum(spare), sum(rows) + sum(spare)) if packed else (lens[0], rows[0])
    lead = () if packed else (b,)
    mk = lambda t, h: torch.randn(lead + (t, h, d), generator=gen).to(dt)  # noqa: E731
    q, k, v = mk(n, hq) * hot, mk(m, hkv), mk(m, hkv)
    if poison:                                              # the last rows are not finite: whoever does not see them is as before
        at = slice(-3, None)
        k[..., at, :, :], v[..., at, :, :] = math.nan, math.inf
        v[..., -2, :, :] = -math.inf
        v[..., -1, :, :] = math.nan
    q_at = [spare[0] + sum(lens[:i]) for i in range(b + 1)]
    k_at = [spare[0] + sum(rows[:i]) for i in range(b + 1)]
    int32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    qd, kd, vd = (_laid_out(x, layout) for x in (q, k, v))
    od = _laid_out(torch.full(lead + (n, hq, d), 7.0, dtype=dt), out_layout)
    lse = torch.full((hq, n) if packed else (b, hq, n), 7.0).cuda()
    p = B.PromptParams(b, hq, hkv, d, n, m, softmax_scale=scale, dtype=mode)
    if packed:
        got = B.ems_prompt_attention(p, qd, kd, vd, q_start=int32(q_at), k_start=int32(k_at), want_lse=True, out=(od, lse))
    else:
        t = lambda x: x.transpose(1, 2)  # noqa: E731
        got = B.ems_prompt_attention(p, t(qd), t(kd), t(vd), want_lse=True, out=(t(od), lse))
    torch.cuda.synchronize()
    assert got[1] is lse
    o, z, g, rms = od.cpu(), lse.cpu(), hq // hkv, Rms()
    for i in range(b):
        qs, ks = (slice(q_at[i], q_at[i + 1]), slice(k_at[i], k_at[i + 1])) if packed else ((i,), (i,))
        for h in heads or range(hq):
            seen = causal(lens[i], rows[i])
            ki, vi = k[ks][..., h // g, :], v[ks][..., h // g, :]
            fine = torch.ones(lens[i], dtype=torch.bool)
            if poison:
                bad = ~(ki.isfinite().all(1) & vi.isfinite().all(1))
                fine = ~(seen & bad).any(1)
                assert fine.sum() >= lens[i] - 3
                assert not o[qs][~fine, h].isfinite().any()
                seen = seen & ~bad
            ref, zr, bound, zb, var = attention_rows(q[qs][..., h, :], ki, vi, seen, scale or d ** -0.5, dt)
            assert_within(o[qs][fine, h], ref[fine], bound[fine], f"sequence {i}, head {h}")
            assert_within((z[h, qs] if packed else z[i, h])[fine], zr[fine], zb[fine], f"lse of sequence {i}, head {h}")
            rms.add(o[qs][fine, h], ref[fine], var[fine])
    rms.check(mode)
    if packed:                                              # rows of no sequence stay as they are
        for at in (slice(0, q_at[0]), slice(q_at[-1], n)):
            assert (o[at] == 7).all() and (z[:, at] == 7).all()


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("case", [
    dict(lens=[1], hq=1, hkv=1, d=64),
    dict(lens=[1, 1, 1], hq=4, hkv=2, d=128),
    dict(lens=[31], hq=2, hkv=2, d=128),
    dict(lens=[32, 32], hq=3, hkv=1, d=64),
    dict(lens=[65], hq=1, hkv=1, d=128, before=[-20]),
    dict(lens=[64], hq=7, hkv=1, d=64, before=[-64]),
    dict(lens=[77], hq=8, hkv=2, d=128, layout="heads", out_layout="heads"),
    dict(lens=[129, 129], hq=4, hkv=4, d=64, layout="odd", out_layout="odd"),
    dict(lens=[130], hq=8, hkv=2, d=128, layout="odd", out_layout="wide"),
    dict(lens=[300], hq=4, hkv=1, d=128, before=[511], layout="wide"),
    dict(lens=[5], hq=20, hkv=1, d=64, before=[3000]),      # few queries, a long axis
    dict(lens=[3, 3], hq=4, hkv=2, d=128, before=[5000, 5000]),
    dict(lens=[1025], hq=2, hkv=1, d=64, scale=0.3),
    dict(lens=[700], hq=6, hkv=2, d=128),
    dict(lens=[70, 1, 0, 33, 128], hq=4, hkv=2, d=64, packed=True),
    dict(lens=[17, 64, 200], hq=6, hkv=3, d=128, packed=True, before=[100, -30, 7], spare=(5, 9)),
    dict(lens=[0, 40, 0], hq=2, hkv=2, d=64, packed=True, spare=(3, 0), layout="odd", out_layout="odd"),
    dict(lens=[40, 300, 5, 64], hq=7, hkv=1, d=128, packed=True, layout="heads", out_layout="wide", before=[0, 1, 2, 3]),
    dict(lens=[9, 2], hq=4, hkv=2, d=128, packed=True, before=[4000, 2500]),
    dict(lens=[i * 7 % 71 for i in range(100)], hq=4, hkv=2, d=64, packed=True, spare=(2, 1)),     # more sequences than lanes
    dict(lens=[1, 0, 40] * 30, hq=2, hkv=1, d=128, packed=True, before=[0, 5, -3] * 30),
])
def test_prompt_matches_64_bits(case, mode):
    _log("prompt", case, mode)
    _prompt_case(**case, mode=mode)


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_of_many_blocks(d, mode):
    """Enough blocks that each takes 256 query rows, whole and not."""
    _log("prompt of many blocks", d, mode)
    _prompt_case([300] * 8, 16, 16, d, mode)
    _prompt_case([130, 700, 1, 515, 64, 90, 256, 257], 32, 8, d, mode, packed=True, layout="heads")


@pytest.mark.parametrize("mode", [BF16, F32])
def test_prompt_with_large_logits(mode):
    """Weights that change by hundreds of powers of two from row to row: the reference moves, first rows count nothing."""
    _log("prompt with large logits", mode)
    _prompt_case([200, 200], 4, 2, 64, mode, hot=40.0)
    _prompt_case([150], 4, 2, 128, mode, hot=25.0, before=[900])


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("n", [40, 70, 128, 300])
def test_prompt_rows_that_a_query_does_not_see_may_hold_anything(n, mode):
    _log("prompt with rows that are not finite", n, mode)
    _prompt_case([n, n], 4, 2, 128, mode, poison=True)
    _prompt_case([n], 2, 2, 64, mode, poison=True, before=[77])


KINDS = [dict(), dict(poison=True), dict(hot=25.0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f32,d,b,hq,hkv,n,m,choice", CHOICES)
def test_prompt_by_every_choice_of_blocks(f32, d, b, hq, hkv, n, m, choice, kind):
    _log("prompt", f32, d, b, hq, hkv, n, m, choice, kind)
    _prompt_case([n] * b, hq, hkv, d, F32 if f32 else BF16, before=[m - n] * b, heads=sorted({0, hq // 2, hq - 1}), **kind)


# ---- chunks over pages

def _chunk_case(n, lens, hq, hkv, d, ps, mode, new_len=None, masked=0.0, layout="tokens", out_layout="tokens", bad_pages=False, seed=0,
                poison=False, whole_mask=False, hot=1.0, heads=None):
    dt = _dtype(mode)
    gen = torch.Generator().manual_seed(seed)
    b = len(lens)
    new = [min(n, max(0, x)) for x in (new_len or [n] * b)]
    columns = max(1, max(-(-m // ps) for m in lens))
    pool = sum(-(-m // ps) for m in lens) + 3
    table = pages_of(lens, ps, pool, columns, gen)
    kp, vp = (torch.randn((pool, hkv, ps, d), generator=gen).to(dt) for _ in range(2))
    pos = None
    if masked or whole_mask:
        pos = torch.where(torch.rand((pool, hkv, ps), generator=gen) < masked, -1, 5).to(torch.int32)
        if whole_mask:
            pos[:, 0] = -1                                  # a head without a live row
        if poison:                                          # what masked rows hold does not matter
            kp[pos < 0], vp[pos < 0] = math.nan, math.inf
    if bad_pages:
        table[0, 0], table[-1, -1] = -3, pool
    used = torch.zeros((pool, ps), dtype=torch.bool)
    for i, m in enumerate(lens):
        for t in range(-(-m // ps)):
            if 0 <= table[i, t] < pool:
                used[table[i, t], :min(ps, m - t * ps)] = True
    if poison:                                              # nor what is behind a length
        rows = ~used[:, None].expand(pool, hkv, ps)
        kp[rows], vp[rows] = math.nan, math.nan
    q = torch.randn((b, n, hq, d), generator=gen).to(dt) * hot
    t = lambda x: x.transpose(1, 2)  # noqa: E731
    qd, od = t(_laid_out(q, layout)), t(_laid_out(torch.full((b, n, hq, d), 7.0, dtype=dt), out_layout))
    lse = torch.full((b, hq, n), 7.0).cuda()
    int32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    p = B.PagedParams(b, hq, hkv, d, ps, pool, columns, dtype=mode)
    cache = B.PagedCache(p, kp.cuda(), vp.cuda(), table.cuda(), positions=None if pos is None else pos.cuda())
    B.ems_paged_chunk_attention(p, cache, int32(lens), qd, new_len=int32(new_len) if new_len else None, want_lse=True, out=(od, lse))
    torch.cuda.synchronize()
    o, z, g, rms = od.cpu(), lse.cpu(), hq // hkv, Rms()
    safe = table.clamp(0, pool - 1)
    there = (table >= 0) & (table < pool)
    for i, m in enumerate(lens):
        for h in heads or range(hq):
            live = there[i].repeat_interleave(ps)[:m]
            if pos is not None:
                live = live & (gather(pos[..., None], safe[i], h // g, m)[:, 0] >= 0)
            seen = causal(new[i], m) & live[None]
            ref, zr, bound, zb, var = attention_rows(q[i, :new[i], h], gather(kp, safe[i], h // g, m), gather(vp, safe[i], h // g, m),
                                                     seen, d ** -0.5, dt)
            assert_within(o[i, h, :new[i]], ref, bound, f"sequence {i}, head {h}")
            assert_within(z[i, h, :new[i]], zr, zb, f"lse of sequence {i}, head {h}")
            rms.add(o[i, h, :new[i]], ref, var)
            assert (o[i, h, new[i]:] == 7).all() and (z[i, h, new[i]:] == 7).all()
    rms.check(mode)


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("case", [
    dict(n=1, lens=[1], hq=1, hkv=1, d=64, ps=16),
    dict(n=1, lens=[0, 5, 64], hq=4, hkv=2, d=128, ps=16),
    dict(n=4, lens=[4, 3, 0, 130], hq=8, hkv=2, d=128, ps=16),
    dict(n=5, lens=[2000, 31, 777], hq=4, hkv=1, d=64, ps=1),
    dict(n=33, lens=[33, 500], hq=7, hkv=1, d=64, ps=7, new_len=[33, 12]),
    dict(n=64, lens=[300, 40, 64, 0], hq=6, hkv=3, d=128, ps=24, new_len=[64, 50, 0, -2]),
    dict(n=100, lens=[1021], hq=4, hkv=2, d=128, ps=100, layout="odd", out_layout="odd"),
    dict(n=130, lens=[131, 700], hq=2, hkv=2, d=64, ps=128, layout="heads", out_layout="wide", new_len=[500, 129]),
    dict(n=3, lens=[6000, 17, 4096], hq=8, hkv=2, d=128, ps=16),
    dict(n=200, lens=[260, 200], hq=20, hkv=1, d=64, ps=16, masked=0.4),
    dict(n=9, lens=[90, 2500], hq=4, hkv=4, d=128, ps=24, masked=0.8),
    dict(n=70, lens=[300, 70], hq=4, hkv=2, d=64, ps=8, masked=0.3, whole_mask=True),
    dict(n=4, lens=[100, 200], hq=4, hkv=2, d=128, ps=16, bad_pages=True),
    dict(n=60, lens=[100, 200], hq=4, hkv=2, d=64, ps=16, bad_pages=True, masked=0.2),
    dict(n=20, lens=[i * 13 % 97 for i in range(70)], hq=4, hkv=2, d=64, ps=16, new_len=[i * 5 % 23 for i in range(70)]),
    dict(n=20, lens=[i * 13 % 97 for i in range(70)], hq=4, hkv=2, d=128, ps=7),
])
def test_chunk_matches_64_bits(case, mode):
    _log("chunk", case, mode)
    _chunk_case(**case, mode=mode)


@pytest.mark.parametrize("mode", [BF16, F32])
def test_chunk_rows_that_take_no_part_may_hold_anything(mode):
    _log("chunk with rows that are not finite", mode)
    _chunk_case(40, [300, 64, 41, 0], 4, 2, 128, 16, mode, masked=0.4, poison=True)
    _chunk_case(3, [2100, 700], 4, 2, 64, 24, mode, masked=0.9, poison=True)
    _chunk_case(200, [333, 200], 8, 2, 64, 16, mode, poison=True)


def test_chunks_of_one_token_are_the_attention_of_one_token():
    """One token a sequence: the same as ems_paged_attention, up to the weights' rounding to 16 bits."""
    gen = torch.Generator().manual_seed(3)
    b, hq, h, d, ps = 5, 8, 2, 128, 16
    lens = [1, 17, 300, 64, 1000]
    pool = sum(-(-m // ps) for m in lens) + 2
    for mode in (BF16, F32):
        p = B.PagedParams(b, hq, h, d, ps, pool, 63, dtype=mode)
        kp, vp = (torch.randn((pool, h, ps, d), generator=gen).to(_dtype(mode)).cuda() for _ in range(2))
        cache = B.PagedCache(p, kp, vp, pages_of(lens, ps, pool, 63, gen).cuda())
        n = torch.tensor(lens, dtype=torch.int32).cuda()
        q = torch.randn((b, hq, d), generator=gen).to(_dtype(mode)).cuda()
        one, z1 = B.ems_paged_attention(p, cache, n, q, want_lse=True)
        many, zn = B.ems_paged_chunk_attention(p, cache, n, q[:, :, None], want_lse=True)
        assert (z1 - zn[..., 0]).abs().max() < 1e-5
        off = (one.double() - many[:, :, 0].double()).norm() / one.double().norm()
        assert off < (2.0 ** -7 if mode == BF16 else 1e-5), off


@pytest.mark.parametrize("kind", [dict(), dict(masked=0.3, poison=True), dict(hot=25.0), dict(hot=25.0, masked=0.9)])
@pytest.mark.parametrize("f32,d,b,hq,hkv,n,m,choice", CHUNK_CHOICES)
def test_chunk_by_every_choice_of_blocks(f32, d, b, hq, hkv, n, m, choice, kind):
    _log("chunk", f32, d, b, hq, hkv, n, m, choice, kind)
    lens = [max(n, m - 150 * i) for i in range(b)]
    _chunk_case(n, lens, hq, hkv, d, 16, F32 if f32 else BF16, heads=sorted({0, hq // 2, hq - 1}), **kind)


# ---- addresses that 32 bits do not hold

def test_prompt_with_sequences_far_apart():
    gen = torch.Generator().manual_seed(4)
    n, h, d, far = 300, 2, 128, (1 << 31) + 512             # elements from sequence to sequence: 4 GiB and some
    p = B.PromptParams(2, h, h, d, n, n)
    near = [torch.randn((2, h, n, d), generator=gen).to(torch.bfloat16).cuda() for _ in range(3)]
    want, z = B.ems_prompt_attention(p, *near, want_lse=True)
    apart = []
    for x in near + [torch.zeros_like(want)]:
        apart.append(torch.empty(far + n * h * d, dtype=torch.bfloat16, device="cuda").as_strided((2, h, n, d), (far, d, h * d, 1)))
        apart[-1].copy_(x)
    got, zg = B.ems_prompt_attention(p, *apart[:3], want_lse=True, out=(apart[3], torch.empty_like(z)))
    assert torch.equal(got, want) and torch.equal(zg, z)


@pytest.mark.parametrize("n", [3, 200])
def test_chunks_of_a_large_pool(n):
    """Pages whose bytes are past 2^32 give what pages at the pool's beginning do."""
    gen = torch.Generator().manual_seed(5)
    b, hq, h, d, ps, pool = 2, 8, 2, 128, 16, 1 << 20       # 8 GiB of keys
    lens = torch.tensor([700, 333], dtype=torch.int32).cuda()
    low = torch.randperm(88, generator=gen).view(2, 44).to(torch.int32).cuda()
    q = torch.randn((b, hq, n, d), generator=gen).to(torch.bfloat16).cuda()
    few = B.PagedParams(b, hq, h, d, ps, 88, 44)
    kp, vp = (torch.randn((88, h, ps, d), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    pos = torch.where(torch.rand((88, h, ps), generator=gen) < 0.2, -1, 0).to(torch.int32).cuda()
    many = B.PagedParams(b, hq, h, d, ps, pool, 44)
    big = [torch.empty((pool,) + x.shape[1:], dtype=x.dtype, device="cuda") for x in (kp, vp, pos)]
    for x, y in zip(big, (kp, vp, pos)):
        x[-88:] = y
    for i in (2, 3):                                        # without and with positions
        mask = lambda x: x if i == 3 else None  # noqa: E731
        want = B.ems_paged_chunk_attention(few, B.PagedCache(few, kp, vp, low, positions=mask(pos)), lens, q)
        got = B.ems_paged_chunk_attention(many, B.PagedCache(many, big[0], big[1], low + (pool - 88), positions=mask(big[2])), lens, q)
        assert torch.equal(got, want)


# ---- graphs

def test_graphs_that_share_a_workspace():
    """Two captured calls whose blocks share tiles, with one workspace, replayed in turn, eager calls between them."""
    gen = torch.Generator().manual_seed(6)
    pp, p = B.PromptParams(1, 4, 4, 128, 40, 3000), B.PagedParams(1, 4, 4, 128, 16, 200, 188)
    need = max(B.ems_prompt_workspace_bytes(pp), B.ems_paged_chunk_workspace_bytes(p, 50))
    assert B.ems_prompt_workspace_bytes(pp) > 0 and B.ems_paged_chunk_workspace_bytes(p, 50) > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    q, k, v, qc = (torch.zeros((1, 4, m, 128), dtype=torch.bfloat16, device="cuda") for m in (40, 3000, 3000, 50))
    table = torch.randperm(200, generator=gen)[:188].view(1, 188).to(torch.int32).cuda()
    cache = B.PagedCache(p, *(torch.randn((200, 4, 16, 128), generator=gen).to(torch.bfloat16).cuda() for _ in range(2)), table)
    lens = torch.tensor([2999], dtype=torch.int32).cuda()
    outs = [torch.zeros_like(q), torch.zeros_like(qc)]
    calls = [lambda o, w: B.ems_prompt_attention(pp, q, k, v, ws=w, out=(o, None)),
             lambda o, w: B.ems_paged_chunk_attention(p, cache, lens, qc, ws=w, out=(o, None))]
    other = torch.empty_like(ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for call, o in zip(calls, outs):
            call(o, ws)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graphs = []
    for call, o in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(o, ws)
        graphs.append(g)
    for _ in range(4):
        for t in (q, k, v, qc):
            t.copy_(torch.randn(t.shape, generator=gen).to(torch.bfloat16))
        want = [torch.full_like(o, 5.0) for o in outs]
        for call, o in zip(calls, want):
            call(o, other)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for got, ref in zip(outs, want):
            assert torch.equal(got, ref)


@pytest.mark.parametrize("mode", [BF16, F32])
def test_prompt_of_large_values(mode):
    """Values of 2^69 and logits that rise from row to row: sums that stay in 32 bits."""
    gen = torch.Generator().manual_seed(7)
    n, d = 700, 128
    q, k, v = (torch.randn((1, 2, n, d), generator=gen).to(_dtype(mode)) for _ in range(3))
    v = (torch.sign(v) * 2.0 ** 69).to(v.dtype)
    q = q * 8
    p = B.PromptParams(1, 2, 2, d, n, n, dtype=mode)
    out = B.ems_prompt_attention(p, q.cuda(), k.cuda(), v.cuda()).cpu()
    for h in range(2):
        ref, _, bound, _, _ = attention_rows(q[0, h], k[0, h], v[0, h], causal(n, n), d ** -0.5, _dtype(mode))
        assert_within(out[0, h], ref, bound, f"head {h}")
