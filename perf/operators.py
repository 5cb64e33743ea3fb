"""The operators of a generation from cached keys and values, as cases that can be timed and compared.

  append    ems_paged_append: new keys and values go into a paged cache, the position rotation is
            applied on the way (to the queries that come with them too)
  attend    ems_paged_attention: one new token per sequence against its pages
  compact   ems_decode_attention: one new token against the compressed cache, whose entries are
            shared by the tokens that were merged (the state that ems_decode_step keeps)

With `own` false `run` computes each in elementary torch operations, in 32 bits (rotation angles in
64), rounded once.  `exact` does it in 64 bits, one sequence at a time.

Inputs: attention mass in real prompts is heavy-tailed, so keys carry an exponentially distributed
component along a direction that the queries share, which makes the weights a power law.  Pages are
handed out in no order, as an allocator leaves them after some time of serving.
"""
import math

import torch

own = False

MASKED = -1          # position of a row that takes no part


def _append(name, batch, q_heads, kv_heads, head_dim, page_size, new, start, rot, *, packed=True, ragged=False,
            interleaved=False, expanded=False, f32=False, with_q=True):
    return dict(name=name, kind="append", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_size=page_size, new=new, start=start, rot=rot, packed=packed, ragged=ragged,
                interleaved=interleaved, expanded=expanded, f32=f32, with_q=with_q, salt=1)


def _attend(name, batch, q_heads, kv_heads, head_dim, page_size, length, *, ragged=False, evicted=0.0, f32=False,
            lse=False, packed=False):
    return dict(name=name, kind="attend", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_size=page_size, length=length, ragged=ragged, evicted=evicted, f32=f32, lse=lse, packed=packed,
                salt=1)


def _compact(name, batch, q_heads, kv_heads, head_dim, budget, window, merge_ratio, *, f32=False, lse=False):
    return dict(name=name, kind="compact", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                budget=budget, window=window, merge_ratio=merge_ratio, f32=f32, lse=lse, salt=1)


def listed():
    return [
        # one sequence, one generated token: a launch and its latency are all there is
        _append("append_one", 1, 32, 8, 128, 16, 1, 77, 128),
        # a full serving batch, one token each
        _append("append_batch", 256, 32, 8, 128, 16, 1, 100, 128),
        # whole prompts straight from the projection (queries, keys and values side by side in every row)
        _append("append_prompt", 4, 32, 8, 128, 16, 8192, 0, 128),
        # a padded batch of prompts of odd lengths, half of the smaller head rotated, neighbouring elements
        # paired, pages that are no power of two, float32
        _append("append_padded", 7, 6, 2, 64, 24, 1021, 13, 32, ragged=True, interleaved=True, f32=True),
        # the expansion of a compressed cache (its rows are rotated already; evicted ones come with their
        # position -1, other ones for every head) becomes the start of a paged generation
        _append("append_expanded", 4, 32, 8, 128, 16, 3040, 0, 0, packed=False, expanded=True, with_q=False),
        # a short context of one sequence, every query head with keys of its own
        _attend("attend_1k", 1, 4, 4, 64, 16, 1024),
        # the longest context of the workloads, one sequence: eight heads have to fill the chip
        _attend("attend_128k", 1, 32, 8, 128, 16, 131072, lse=True),
        # a serving batch of very different lengths, the longest 32768
        _attend("attend_ragged", 64, 32, 8, 128, 16, 32768, ragged=True),
        # many sequences on expanded compressed caches, three rows in ten evicted, head by head
        _attend("attend_evicted", 128, 32, 8, 128, 32, 1500, evicted=0.3, packed=True),
        # float32, the mode that checks the other: odd sizes all round
        _attend("attend_f32", 3, 21, 3, 64, 24, 5003, ragged=True, evicted=0.1, f32=True, lse=True),
        # generation from the compact cache: the 32K workload's budget, four sequences
        _compact("compact_b128", 4, 32, 8, 128, 128, 64, 0.5),
        # the 128K workload's budget, a batch of sequences
        _compact("compact_b2048", 32, 32, 8, 128, 2048, 64, 0.5, lse=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "compact"])
    while True:
        head_dim = rng.choice([64, 128, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
        f32 = rng.random() < 0.15
        page = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100, 128, 256])
        if kind == "append":
            group = rng.choice([1, 2, 3, 4, 4, 7, 8])
            expanded = rng.random() < 0.2
            new = rng.choice([1, 1, _log_int(rng, 2, 16384)])
            c = _append("", _log_int(rng, 1, 256), kv_heads * group, kv_heads, head_dim, page, new,
                        rng.choice([0, _log_int(rng, 1, 300)]),
                        0 if expanded else rng.choice([head_dim, head_dim, head_dim // 2, 16]),
                        packed=not expanded and rng.random() < 0.7, ragged=new > 1 and rng.random() < 0.5,
                        interleaved=rng.random() < 0.3, expanded=expanded, f32=f32,
                        with_q=not expanded and rng.random() < 0.7)
        elif kind == "attend":
            group = rng.choice([1, 2, 3, 4, 4, 7, 8, 16, 20])
            c = _attend("", _log_int(rng, 1, 256), kv_heads * group, kv_heads, head_dim, page,
                        _log_int(rng, 1, 131072), ragged=rng.random() < 0.5, evicted=rng.choice([0.0, 0.0, 0.1, 0.6]),
                        f32=f32, lse=rng.random() < 0.5, packed=rng.random() < 0.5)
        else:
            group = rng.choice([1, 2, 4, 4, 8])
            window = rng.choice([16, 32, 33, 64])
            c = _compact("", _log_int(rng, 1, 64), kv_heads * group, kv_heads, head_dim, window + _log_int(rng, 16, 4096),
                         window, rng.choice([0.0, 0.25, 0.5, 0.5, 1.0, 2.0]), f32=f32, lse=rng.random() < 0.5)
        del c["name"]
        c["salt"] = rng.randint(1, 1 << 20)
        # no more bytes than the largest listed case of its kind
        most = {"append": 0.9e9, "attend": 4.0e9, "compact": 3.0e8}[kind]
        if work(c)["bytes"] <= most:
            return c


# ---- sizes that follow from a case alone

def _spread(c, most):
    """`batch` lengths in 1..most: all the longest, or spread evenly with one of them the longest."""
    b = c["batch"]
    if not c["ragged"]:
        return [most] * b
    u = [((i + 1) * 2654435761 + c["salt"] * 40503) % 4294967296 / 4294967296 for i in range(b)]
    u[c["salt"] % b] = 1.0
    return [max(1, round(most * x)) for x in u]


def _elem_bytes(c):
    return 4 if c["f32"] else 2


def _table_size(c):
    n_imp = c["budget"] - c["window"]
    n_tbm = int(math.floor(c["merge_ratio"] * c["budget"]))
    return n_imp, n_tbm, n_imp + n_tbm + c["window"]


def _geometry(c):
    """Lengths of the sequences (append: new tokens), first slots, pages of each, columns of the table."""
    if c["kind"] == "append":
        lens = _spread(c, c["new"])
        first = [(c["start"] + 5 * i * (c["start"] > 0)) % (2 * c["start"] + 1) for i in range(c["batch"])]
    else:
        lens = _spread(c, c["length"])
        first = [0] * c["batch"]
    pages = [-(-(s + n) // c["page_size"]) for s, n in zip(first, lens)]
    return lens, first, pages, max(pages)


def work(case):
    """Inputs read once, outputs written once."""
    c = case
    e, d, h, hq = _elem_bytes(c), c["head_dim"], c["kv_heads"], c["q_heads"]
    row = d * e
    if c["kind"] == "compact":
        n_imp, n_tbm, t = _table_size(c)
        unit = 2 * row * (c["budget"] + 1) + 8 * t + 4 * c["budget"]
        heads = 2 * row + (4 if c["lse"] else 0)
        return {"bytes": c["batch"] * (h * unit + hq * heads), "flops": 4.0 * d * c["batch"] * hq * (c["budget"] + 1)}
    lens, _, pages, _ = _geometry(c)
    n = sum(lens)
    if c["kind"] == "append":
        heads = 2 * h + (hq if c["with_q"] else 0)
        turned = h + (hq if c["with_q"] else 0)
        pos = (8 * h * n) if c["expanded"] else 0
        return {"bytes": 2 * row * heads * n + pos + 4 * sum(pages) + 8 * c["batch"], "flops": 3.0 * c["rot"] * turned * n}
    pos = 4 * h * n if c["evicted"] else 0
    live = (1 - c["evicted"]) * n                  # an evicted row need not be read
    return {"bytes": 2 * row * h * live + pos + 4 * sum(pages) + c["batch"] * (4 + hq * (2 * row + (4 if c["lse"] else 0))),
            "flops": 4.0 * d * hq * live}


# ---- inputs

def _dtype(c):
    return torch.float32 if c["f32"] else torch.bfloat16


def _direction(c, gen):
    u = torch.randn((c["kv_heads"], 1, c["head_dim"]), device="cuda", generator=gen)
    return u / u.norm(dim=-1, keepdim=True)


def _rows(c, lead, n, u, gen, keys):
    """[lead, kv_heads, n, D] keys or values, made in pieces of at most half a gigabyte."""
    h, d = c["kv_heads"], c["head_dim"]
    out = torch.empty((lead, h, n, d), dtype=_dtype(c), device="cuda")
    step = max(1, (1 << 27) // (h * n * d))
    for i in range(0, lead, step):
        m = min(step, lead - i)
        x = torch.randn((m, h, n, d), device="cuda", generator=gen)
        if keys:
            heavy = torch.empty((m, h, n, 1), device="cuda").exponential_(1.0, generator=gen)
            x += 0.25 * math.sqrt(d) * heavy * u
        out[i:i + m] = x
    return out


def _queries(c, u, gen):
    """[B, Hq, D]; in a packed case a view of the projection's row, which holds keys and values behind them."""
    b, hq, h, d = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    q = torch.randn((b, hq, d), device="cuda", generator=gen)
    q = (q.view(b, h, hq // h, d) + 4.0 * u).view(b, hq, d).to(_dtype(c))
    if not c.get("packed"):
        return q
    wide = torch.zeros((b, (hq + 2 * h) * d), dtype=_dtype(c), device="cuda")
    wide[:, :hq * d] = q.reshape(b, hq * d)
    return wide[:, :hq * d].view(b, hq, d)


def _pages(c, pages, columns, gen):
    """A pool with a few spare pages and the table of each sequence's; unused columns hold -1."""
    pool = sum(pages) + 5
    order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((c["batch"], columns), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    return pool, table


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "compact":
        _prepare_compact(c, s, gen)
    else:
        b, h, d, ps = c["batch"], c["kv_heads"], c["head_dim"], c["page_size"]
        lens, first, pages, columns = _geometry(c)
        pool, s["table"] = _pages(c, pages, columns, gen)
        u = _direction(c, gen)
        s["k_pages"] = _rows(c, pool, ps, u, gen, True)
        s["v_pages"] = _rows(c, pool, ps, u, gen, False)
        s["pos_pages"] = None
        int32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        if c["kind"] == "append":
            _prepare_append(c, s, gen, lens, first, int32)
        else:
            s["lens"] = int32(lens)
            s["q"] = _queries(c, u, gen)
            if c["evicted"]:
                gone = torch.rand((pool, h, ps), device="cuda", generator=gen) < c["evicted"]
                at = torch.randint(0, 1 << 20, (pool, h, ps), device="cuda", generator=gen, dtype=torch.int32)
                s["pos_pages"] = torch.where(gone, MASKED, at)
        if own:
            from paper_2412_08521_amd import binding as B
            p = B.PagedParams(b, c["q_heads"], h, d, ps, pool, columns, dtype=B.EMS_F32 if c["f32"] else B.EMS_BF16)
            s["p"] = p
            s["cache"] = B.PagedCache(p, s["k_pages"], s["v_pages"], s["table"], positions=s["pos_pages"])
            if c["kind"] == "attend":
                s["ws"] = torch.empty(max(B.ems_paged_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
                s["out"] = torch.empty((b, c["q_heads"], d), dtype=_dtype(c), device="cuda")
                s["lse"] = torch.empty((b, c["q_heads"]), device="cuda") if c["lse"] else None
    torch.cuda.synchronize()
    return s


def _prepare_append(c, s, gen, lens, first, int32):
    b, hq, h, d, n = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["new"]
    dt = _dtype(c)
    nq = hq if c["with_q"] else 0
    if c["packed"]:
        # [B, N, (Hq + 2 Hkv) D], as the projection leaves it; heads and tokens change places in the view only
        x = torch.randn((b, n, nq + 2 * h, d), device="cuda", generator=gen).to(dt)
        views = [x[:, :, i:j].transpose(1, 2) for i, j in ((0, nq), (nq, nq + h), (nq + h, nq + 2 * h))]
    else:
        views = [torch.randn((b, m, n, d), device="cuda", generator=gen).to(dt) for m in (nq, h, h)]
    s["q"], s["k"], s["v"] = (views[0] if nq else None), views[1], views[2]
    s["start"] = int32(first)
    s["new_len"] = int32(lens) if c["ragged"] else None
    # 10000^(-2i/rot), the usual frequencies; far positions too (a sequence whose earlier tokens left the cache)
    s["inv_freq"] = None
    if c["rot"]:
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().cuda()
    s["positions"] = None
    if c["expanded"]:
        gone = torch.rand((b, h, n), device="cuda", generator=gen) < 0.3
        at = torch.arange(n, device="cuda", dtype=torch.int32) * 41
        s["positions"] = torch.where(gone, MASKED, at)
        s["pos_pages"] = torch.full(s["k_pages"].shape[:3], MASKED, dtype=torch.int32, device="cuda")
    elif c["salt"] % 2 == 0:
        s["positions"] = (s["start"][:, None] + 100000 + torch.arange(n, device="cuda", dtype=torch.int32)[None]).contiguous()
    s["q_out"] = torch.zeros((b, hq, n, d), dtype=dt, device="cuda") if nq else None
    s["len_out"] = torch.zeros(b, dtype=torch.int32, device="cuda")


def _prepare_compact(c, s, gen):
    """The state of a compressed cache: budget rows per head (entries, then the window), and a table of tokens
    that point to them, each with its own key norm.  Four in ten of the merged tokens have been evicted."""
    b, h, hq, d, nb, w = c["batch"], c["kv_heads"], c["q_heads"], c["head_dim"], c["budget"], c["window"]
    n_imp, n_tbm, t = _table_size(c)
    u = _direction(c, gen)
    s["k_cache"] = _rows(c, b, nb + 1, u, gen, True)
    s["v_cache"] = _rows(c, b, nb + 1, u, gen, False)
    s["row_norm"] = s["k_cache"][:, :, :nb].float().norm(dim=-1).contiguous()
    dest = torch.randint(0, n_imp, (b, h, n_tbm), device="cuda", generator=gen)
    dest = torch.where(torch.rand((b, h, n_tbm), device="cuda", generator=gen) < 0.4, -1, dest)
    at = torch.arange(nb, device="cuda").expand(b, h, nb)
    rows = torch.cat([at[:, :, :n_imp], dest, at[:, :, n_imp:]], dim=2)
    s["tok_row"] = rows.to(torch.int32).contiguous()
    share = torch.ones((b, h, t), device="cuda")
    share[:, :, n_imp:n_imp + n_tbm] = 0.6 + 0.6 * torch.rand((b, h, n_tbm), device="cuda", generator=gen)
    s["tok_norm"] = (share * s["row_norm"].gather(2, rows.clamp(min=0))).contiguous()
    s["q"] = _queries(c, u, gen)
    s["k_new"] = _rows(c, b, 1, u, gen, True)[:, :, 0].contiguous()
    s["v_new"] = _rows(c, b, 1, u, gen, False)[:, :, 0].contiguous()
    if own:
        from paper_2412_08521_amd import binding as B
        p = B.EmsParams(b, hq, h, d, nb + n_tbm + 1, w, nb, merge_ratio=c["merge_ratio"],
                        dtype=B.EMS_F32 if c["f32"] else B.EMS_BF16)
        st = B.DecodeState(p, s["k_cache"], s["v_cache"])
        for name in ("row_norm", "tok_row", "tok_norm"):
            getattr(st, name).copy_(s[name])
        s["p"], s["state"] = p, st
        s["ws"] = torch.empty(max(B.ems_decode_attention_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((b, hq, d), dtype=_dtype(c), device="cuda")
        s["lse"] = torch.empty((b, hq), device="cuda") if c["lse"] else None


# ---- one pass

def run(state):
    s = state
    c = s["case"]
    if own:
        return _run_own(c, s)
    if c["kind"] == "append":
        return _plain_append(c, s)
    return _plain_attend(c, s) if c["kind"] == "attend" else _plain_compact(c, s)


def _run_own(c, s):
    from paper_2412_08521_amd import binding as B
    if c["kind"] == "append":
        q_out = B.ems_paged_append(s["p"], s["cache"], s["start"], s["k"], s["v"], positions=s["positions"],
                                   new_len=s["new_len"], inv_freq=s["inv_freq"], interleaved=c["interleaved"],
                                   q=s["q"], q_out=s["q_out"], len_out=s["len_out"])
        return s["k_pages"], s["v_pages"], s["pos_pages"], q_out, s["len_out"]
    if c["kind"] == "attend":
        return B.ems_paged_attention(s["p"], s["cache"], s["lens"], s["q"], want_lse=c["lse"], ws=s["ws"],
                                     out=(s["out"], s["lse"]))
    return B.ems_decode_attention(s["p"], s["state"], s["q"], s["k_new"], s["v_new"], want_lse=c["lse"], ws=s["ws"],
                                  out=(s["out"], s["lse"]))


def _turned(x, cos, sin, rot, interleaved):
    """x [B, H, N, D] in 32 bits, cos and sin [B, H or 1, N, rot / 2]."""
    a, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a0, a1 = a[..., 0::2], a[..., 1::2]
        out = torch.stack((a0 * cos - a1 * sin, a1 * cos + a0 * sin), dim=-1).flatten(-2)
    else:
        a0, a1 = a[..., :rot // 2], a[..., rot // 2:]
        out = torch.cat((a0 * cos - a1 * sin, a1 * cos + a0 * sin), dim=-1)
    return torch.cat((out, rest), dim=-1)


def _plain_append(c, s):
    b, n, ps = c["batch"], c["new"], c["page_size"]
    dt = _dtype(c)
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    slot = s["start"][:, None] + i[None]                                          # [B, N]
    live = i[None] < (s["new_len"][:, None] if s["new_len"] is not None else n)
    live = live.expand(b, n)
    pos = s["positions"] if s["positions"] is not None else slot
    if pos.dim() == 2:
        pos = pos[:, None]                                                        # [B, H or 1, N]
    k, q = s["k"], s["q"]
    if c["rot"]:
        angle = pos[..., None].double() * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        k = _turned(k.float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
        if q is not None:
            g = c["q_heads"] // c["kv_heads"]
            if cos.shape[1] > 1:
                cos, sin = cos.repeat_interleave(g, 1), sin.repeat_interleave(g, 1)
            q = _turned(q.float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    bi, ni = live.nonzero(as_tuple=True)
    page = s["table"][bi, (slot[bi, ni] // ps).long()].long()
    at = (slot[bi, ni] % ps).long()
    s["k_pages"][page, :, at] = k[bi, :, ni]
    s["v_pages"][page, :, at] = s["v"][bi, :, ni]
    if s["pos_pages"] is not None:
        s["pos_pages"][page, :, at] = pos.expand(b, c["kv_heads"], n)[bi, :, ni]
    if q is not None:
        s["q_out"][bi, :, ni] = q[bi, :, ni]
    s["len_out"].copy_(s["start"] + live.sum(1, dtype=torch.int32))
    return s["k_pages"], s["v_pages"], s["pos_pages"], s["q_out"], s["len_out"]


def _softmax_rows(logits, live, v):
    """logits, live [..., G, L] and v [..., L, D], masked rows of v zero -> output and log-sum-exp; an empty row gives
    zeros and -inf."""
    logits = torch.where(live, logits, -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = (logits - top).exp()
    total = p.sum(dim=-1, keepdim=True)
    out = torch.where(total > 0, (p @ v) / total, 0.0)
    return out, (top + total.log())[..., 0]


def _plain_attend(c, s):
    b, hq, h, d, ps = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_size"]
    g, scale = hq // h, d ** -0.5
    columns = s["table"].shape[1]
    lens = _geometry(c)[0]
    out, lse = [], []
    # as many sequences at a time as about two gigabytes hold, cut to their longest
    step = max(1, (1 << 29) // (h * columns * ps * d))
    for b0 in range(0, b, step):
        b1 = min(b, b0 + step)
        n = -(-max(lens[b0:b1]) // ps)
        table = s["table"][b0:b1, :n]
        m, width = b1 - b0, n * ps
        gather = lambda x: x[table.clamp(min=0).long()].transpose(1, 2).reshape((m, h, width) + tuple(x.shape[3:]))  # noqa: E731
        live = (torch.arange(width, device="cuda") < s["lens"][b0:b1, None])[:, None].expand(m, h, width)
        if s["pos_pages"] is not None:
            live = live & (gather(s["pos_pages"]) >= 0)
        k = gather(s["k_pages"]).float()
        logits = (s["q"][b0:b1].float().reshape(m, h, g, d) @ k.transpose(-1, -2)) * scale
        del k
        v = torch.where(live[..., None], gather(s["v_pages"]).float(), 0.0)
        o, z = _softmax_rows(logits, live[:, :, None], v)
        out.append(o.reshape(m, hq, d).to(_dtype(c)))
        lse.append(z.reshape(m, hq))
    out = torch.cat(out)
    return (out, torch.cat(lse)) if c["lse"] else out


def _plain_compact(c, s):
    b, hq, h, d = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    g = hq // h
    row = s["tok_row"]
    live, at = row >= 0, row.clamp(min=0).long()
    norm = s["row_norm"].gather(2, at)
    factor = torch.where(norm > 0, s["tok_norm"] / norm, 0.0)
    take = lambda x: x.gather(2, at[..., None].expand(*at.shape, d)).float()  # noqa: E731
    k = torch.cat((take(s["k_cache"]) * factor[..., None], s["k_new"][:, :, None].float()), dim=2)
    live = torch.cat((live, torch.ones_like(live[:, :, :1])), dim=2)
    logits = (s["q"].float().view(b, h, g, d) @ k.transpose(-1, -2)) * d ** -0.5
    v = torch.cat((take(s["v_cache"]), s["v_new"][:, :, None].float()), dim=2)
    o, z = _softmax_rows(logits, live[:, :, None], torch.where(live[..., None], v, 0.0))
    out = o.view(b, hq, d).to(_dtype(c))
    return (out, z.view(b, hq)) if c["lse"] else out


# ---- the same in 64 bits, from the definitions

def exact(case, seed):
    """None in the place of positions and lengths."""
    c = case
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _exact_append(c, s)
    b, hq, h, d = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    g = hq // h
    out = torch.zeros((b, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq), -math.inf, dtype=torch.float64, device="cuda")
    lens = _geometry(c)[0] if c["kind"] == "attend" else None
    for i in range(b):
        for j in range(h):
            if c["kind"] == "attend":
                n = lens[i]
                pages = s["table"][i, :-(-n // c["page_size"])].long()
                k, v = (s[x][pages, j].reshape(-1, d)[:n].double() for x in ("k_pages", "v_pages"))
                if s["pos_pages"] is not None:
                    keep = s["pos_pages"][pages, j].reshape(-1)[:n] >= 0
                    k, v = k[keep], v[keep]
            else:
                keep = s["tok_row"][i, j] >= 0
                r = s["tok_row"][i, j][keep].long()
                length = s["row_norm"][i, j][r].double()
                ratio = torch.where(length > 0, s["tok_norm"][i, j][keep].double() / length, 0.0)
                k = torch.vstack([s["k_cache"][i, j, r].double() * ratio[:, None], s["k_new"][i, j].double()[None]])
                v = torch.vstack([s["v_cache"][i, j, r].double(), s["v_new"][i, j].double()[None]])
            if len(k) == 0:
                continue
            x = s["q"][i, j * g:(j + 1) * g].double() @ k.T / math.sqrt(d)
            z = torch.logsumexp(x, dim=1)
            lse[i, j * g:(j + 1) * g] = z
            out[i, j * g:(j + 1) * g] = (x - z[:, None]).exp() @ v
    return (out, lse) if c["lse"] else out


def _exact_append(c, s):
    d, h, hq, ps, rot, half = c["head_dim"], c["kv_heads"], c["q_heads"], c["page_size"], c["rot"], c["rot"] // 2
    lens, first, _, _ = _geometry(c)
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    qo = s["q_out"].double() if s["q_out"] is not None else None
    # columns of the first and of the second element of every pair
    pair = torch.arange(half, device="cuda")
    one, two = (2 * pair, 2 * pair + 1) if c["interleaved"] else (pair, pair + half)
    for i in range(c["batch"]):
        n = lens[i]
        slot = torch.arange(first[i], first[i] + n, device="cuda")
        if s["positions"] is None:
            pos = slot[None]
        elif s["positions"].dim() == 2:
            pos = s["positions"][i:i + 1, :n]
        else:
            pos = s["positions"][i, :, :n]
        page, at = s["table"][i].long()[slot // ps], slot % ps
        for src, heads in (("k", h), ("q", hq)):
            if s[src] is None:
                continue
            x = s[src][i, :, :n].double()
            if rot:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                                   pos[..., None].double() * s["inv_freq"].double())
                if turn.shape[0] > 1:
                    turn = turn.repeat_interleave(heads // h, 0)
                z = torch.complex(x[..., one], x[..., two]) * turn
                x = x.clone()
                x[..., one], x[..., two] = z.real, z.imag
            if src == "k":
                kp[page, :, at] = x.transpose(0, 1)
            else:
                qo[i, :, :n] = x
        vp[page, :, at] = s["v"][i, :, :n].double().transpose(0, 1)
    return kp, vp, None, qo, None
