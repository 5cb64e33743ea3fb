"""The operators of a prompt and of a chunk of it, and of a paged cache in 8 bits, as cases that can be timed and compared.

  prompt    ems_prompt_attention: causal attention of whole prompts with grouped heads, the sequences of a batch side by
            side or packed one after the other; the log-sum-exp of its rows is what the score of a prompt starts from
  chunk     ems_paged_chunk_attention: the newest tokens of every sequence against its pages, theirs among them
  store8    ems_quant_append, ems_quant_read: new keys and values are rotated and go into a paged cache as 8-bit numbers
            (e4m3, a power of two for every row), and the sequences' rows are read back for the attention of a chunk
  attend8   ems_quant_attention: one new token per sequence against its 8-bit pages

With `own` false `run` computes each in elementary torch operations, in 32 bits (rotation angles in 64), rounded once.
`exact` does it in 64 bits, one sequence at a time.

Inputs: attention mass in real prompts is heavy-tailed, so keys carry an exponentially distributed component along a
direction that the queries share, which makes the weights a power law.  Pages are handed out in no order, as an allocator
leaves them after some time of serving.
"""
import math

import torch

own = False

MASKED = -1          # position of a row that takes no part


def _prompt(name, batch, q_heads, kv_heads, head_dim, length, *, prefix=0, packed=False, ragged=False, f32=False, lse=False):
    return dict(name=name, kind="prompt", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, length=length,
                prefix=prefix, packed=packed, ragged=ragged, f32=f32, lse=lse, salt=1)


def _chunk(name, batch, q_heads, kv_heads, head_dim, page_size, new, length, *, ragged=False, evicted=0.0, f32=False, lse=False):
    return dict(name=name, kind="chunk", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_size=page_size, new=new, length=length, ragged=ragged, evicted=evicted, f32=f32, lse=lse, salt=1)


def _store8(name, batch, q_heads, kv_heads, head_dim, page_size, new, start, rot, *, ragged=False, interleaved=False,
            with_q=True):
    return dict(name=name, kind="store8", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_size=page_size, new=new, start=start, rot=rot, ragged=ragged, interleaved=interleaved, with_q=with_q,
                f32=False, salt=1)


def _attend8(name, batch, q_heads, kv_heads, head_dim, page_size, length, *, ragged=False, evicted=0.0, lse=False):
    return dict(name=name, kind="attend8", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                page_size=page_size, length=length, ragged=ragged, evicted=evicted, lse=lse, f32=False, salt=1)


def listed():
    return [
        # one question of an interactive session: latency
        _prompt("prompt_short", 1, 32, 8, 128, 77),
        # a short prompt, every query head with keys of its own
        _prompt("prompt_1k", 1, 4, 4, 64, 1024, lse=True),
        # a batch of prompts of very different lengths, packed, straight from the projection
        _prompt("prompt_packed", 16, 32, 8, 128, 4096, packed=True, ragged=True),
        # the 32K workload's prompt, with the log-sum-exp that its score starts from
        _prompt("prompt_32k", 1, 32, 8, 128, 32768, lse=True),
        # float32, the mode that checks the other: odd sizes, and keys that the cache of an earlier turn holds already
        _prompt("prompt_f32", 3, 6, 2, 64, 1021, prefix=300, ragged=True, packed=True, f32=True, lse=True),
        # drafts of four tokens each, checked against contexts of very different lengths: few rows, a long axis
        _chunk("chunk_draft", 8, 32, 8, 128, 16, 4, 8192, ragged=True),
        # a chunk of a long prompt
        _chunk("chunk_prompt", 1, 32, 8, 128, 16, 2048, 32768),
        # chunks of odd lengths behind compressed prompts, whose evicted rows are masked head by head
        _chunk("chunk_evicted", 24, 28, 4, 64, 24, 511, 3001, ragged=True, evicted=0.3, lse=True),
        # a chunk of a prompt that follows what the cache holds
        _store8("store8_chunk", 1, 32, 8, 128, 16, 512, 1536, 128),
        # whole prompts of different lengths
        _store8("store8_prompt", 4, 32, 8, 128, 16, 8192, 0, 128, ragged=True),
        # a small batch of short contexts
        _attend8("attend8_1k", 4, 8, 4, 64, 16, 1000, ragged=True),
        # a serving batch of very different lengths, the longest 32768
        _attend8("attend8_ragged", 64, 32, 8, 128, 16, 32768, ragged=True, lse=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "chunk", "chunk", "store8", "attend8"])
    while True:
        head_dim = rng.choice([64, 128, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
        f32 = rng.random() < 0.15
        page = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 100, 128, 256])
        group = rng.choice([1, 2, 3, 4, 4, 7, 8, 20])
        heads = (kv_heads * group, kv_heads, head_dim)
        if kind == "prompt":
            c = _prompt("", _log_int(rng, 1, 64), *heads, _log_int(rng, 1, 32768),
                        prefix=rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]), packed=rng.random() < 0.5,
                        ragged=rng.random() < 0.6, f32=f32, lse=rng.random() < 0.5)
            c["ragged"] = c["ragged"] and c["packed"]
        elif kind == "chunk":
            new = rng.choice([1, _log_int(rng, 2, 16), _log_int(rng, 2, 4096)])
            c = _chunk("", _log_int(rng, 1, 64), *heads, page, new, new + _log_int(rng, 1, 32768) - 1,
                       ragged=rng.random() < 0.5, evicted=rng.choice([0.0, 0.0, 0.1, 0.6]), f32=f32, lse=rng.random() < 0.5)
        elif kind == "store8":
            new = rng.choice([1, _log_int(rng, 2, 8192)])
            c = _store8("", _log_int(rng, 1, 64), *heads, page, new, rng.choice([0, _log_int(rng, 1, 4096)]),
                        rng.choice([0, head_dim, head_dim, head_dim // 2, 16]), ragged=new > 1 and rng.random() < 0.5,
                        interleaved=rng.random() < 0.3, with_q=rng.random() < 0.7)
        else:
            c = _attend8("", _log_int(rng, 1, 256), *heads, page, _log_int(rng, 1, 65536), ragged=rng.random() < 0.5,
                         evicted=rng.choice([0.0, 0.0, 0.1, 0.6]), lse=rng.random() < 0.5)
        del c["name"]
        c["salt"] = rng.randint(1, 1 << 20)
        # no more than the largest listed case of its kind: in work, and in the padded scores that the plain form goes through
        w, most = work(c), {"prompt": 8.9e12, "chunk": 1.1e12, "store8": 1e15, "attend8": 1e15}[kind] * (0.1 if f32 else 1)
        if w["flops"] <= most and w["bytes"] <= {"store8": 5.0e8, "attend8": 2.4e9}.get(kind, 2.0e9) and _scores(c) <= 1.8e10:
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


def _geometry(c):
    """New tokens of every sequence (queries, or rows that are stored), and rows of keys, theirs the last."""
    b = c["batch"]
    if c["kind"] == "prompt":
        new = _spread(c, c["length"])
        before = [(c["prefix"] + 7 * i * (c["prefix"] > 0)) % (2 * c["prefix"] + 1) for i in range(b)] if c["ragged"] else [c["prefix"]] * b
    elif c["kind"] == "chunk":
        rows = _spread(c, c["length"])
        new = [min(n, m) for n, m in zip(_spread({**c, "salt": c["salt"] + 3}, c["new"]), rows)]
        before = [m - n for n, m in zip(new, rows)]
    elif c["kind"] == "store8":
        new = _spread(c, c["new"])
        before = [(c["start"] + 5 * i * (c["start"] > 0)) % (2 * c["start"] + 1) for i in range(b)]
    else:
        new, before = [0] * b, _spread(c, c["length"])
    return new, [n + s for n, s in zip(new, before)]


def _scores(c):
    """Scores of the plain form, which pads every sequence to the longest."""
    new, rows = _geometry(c)
    return c["batch"] * c["q_heads"] * max(max(new), 1) * max(rows) if c["kind"] != "store8" else 0


def work(case):
    """Inputs read once, outputs written once; an evicted row need not be read, a pair that is not seen not be formed."""
    c = case
    e, d, h, hq, b = (4 if c["f32"] else 2), c["head_dim"], c["kv_heads"], c["q_heads"], c["batch"]
    new, rows = _geometry(c)
    q, kv, live = sum(new), sum(rows), 1 - c.get("evicted", 0.0)
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(new, rows))
    lse = 4 * hq * q if c.get("lse") else 0
    table = 4 * sum(-(-m // c["page_size"]) for m in rows) if c["kind"] != "prompt" else 0
    if c["kind"] == "prompt":
        return {"bytes": 2 * d * e * (hq * q + h * kv) + lse + 8 * c["packed"] * (b + 1), "flops": 4.0 * d * hq * pairs}
    if c["kind"] == "chunk":
        pos = 4 * h * kv if c["evicted"] else 0
        return {"bytes": 2 * d * e * (hq * q + h * kv * live) + lse + pos + table + 8 * b, "flops": 4.0 * d * hq * pairs * live}
    if c["kind"] == "store8":
        n_q = hq if c["with_q"] else 0
        # rows that were there are read as bytes, new ones are written as bytes; all of them are written out
        return {"bytes": 2 * h * (q * (2 * d + d + 1) + (kv - q) * (d + 1) + kv * 2 * d) + 4 * n_q * q * d + table + 12 * b,
                "flops": 3.0 * c["rot"] * (h + n_q) * q + 2.0 * h * d * (q + kv)}
    pos = 4 * h * kv if c["evicted"] else 0
    return {"bytes": 2 * h * (d + 1) * kv * live + pos + table + b * (4 + hq * (4 * d + (4 if c["lse"] else 0))),
            "flops": 4.0 * d * hq * kv * live}


# ---- inputs

def _dtype(c):
    return torch.float32 if c["f32"] else torch.bfloat16


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _direction(c, gen):
    u = torch.randn((c["kv_heads"], c["head_dim"]), device="cuda", generator=gen)
    return u / u.norm(dim=-1, keepdim=True)


def _heavy(c, x, u, gen):
    """Keys [.., H, D] from normal numbers x of that shape."""
    weight = torch.empty(x.shape[:-1] + (1,), device="cuda").exponential_(1.0, generator=gen)
    return x + 0.25 * math.sqrt(c["head_dim"]) * weight * u


def _seeking(c, x, u):
    """Queries [.., Hq, D] from normal numbers."""
    h = c["kv_heads"]
    return (x.view(x.shape[:-2] + (h, c["q_heads"] // h, x.shape[-1])) + 4.0 * u[:, None]).view(x.shape)


def _page_rows(c, pool, u, gen, keys):
    """[pool, H, page_size, D] keys or values, made in pieces of at most half a gigabyte."""
    h, d, ps = c["kv_heads"], c["head_dim"], c["page_size"]
    out = torch.empty((pool, h, ps, d), dtype=_dtype(c), device="cuda")
    step = max(1, (1 << 27) // (h * ps * d))
    for i in range(0, pool, step):
        x = torch.randn((min(step, pool - i), ps, h, d), device="cuda", generator=gen)
        out[i:i + step] = (_heavy(c, x, u, gen) if keys else x).transpose(1, 2)
    return out


def _pages(c, rows, gen):
    """A pool with a few spare pages and the table of each sequence's; unused columns hold -1."""
    pages = [-(-m // c["page_size"]) for m in rows]
    pool = sum(pages) + 5
    order = torch.randperm(pool, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((c["batch"], max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    return pool, table


def _quantized(x):
    """Rows [.., D] in 32 bits or more -> their e4m3 numbers and the byte s + 127 of each row's 2^s: the smallest power of
    two, from 2^-126, by which the row's largest modulus is at most 448, the largest e4m3 number."""
    mant, exp = torch.frexp(x.abs().amax(dim=-1))                    # mant in [1/2, 1): 448 = 7/8 2^9
    s = torch.where(mant > 0, exp - 9 + (mant > 0.875).to(exp.dtype), -126).clamp(min=-126)
    return torch.ldexp(x, -s[..., None]).to(torch.float8_e4m3fn), (s + 127).to(torch.uint8)


def _value(code, byte, dtype=torch.float32):
    return torch.ldexp(code.to(dtype), (byte.to(torch.int32) - 127)[..., None])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    u = _direction(c, gen)
    if c["kind"] == "prompt":
        _prepare_prompt(c, s, u, gen)
    else:
        _prepare_paged(c, s, u, gen)
    torch.cuda.synchronize()
    return s


def _prepare_prompt(c, s, u, gen):
    b, hq, h, d, dt = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], _dtype(c)
    new, rows = _geometry(c)
    n, m = (sum(new), sum(rows)) if c["packed"] else (new[0], rows[0])
    lead = () if c["packed"] else (b,)
    rand = lambda count, heads: torch.randn(lead + (count, heads, d), device="cuda", generator=gen)  # noqa: E731
    q, k, v = _seeking(c, rand(n, hq), u), _heavy(c, rand(m, h), u, gen), rand(m, h)
    if c["packed"] and n == m:
        # [T, (Hq + 2 Hkv), D], as the projection leaves it
        x = torch.cat([q, k, v], dim=1).to(dt)
        s["q"], s["k"], s["v"] = x.split([hq, h, h], dim=1)
    elif c["packed"]:
        s["q"], s["k"], s["v"] = q.to(dt), k.to(dt), v.to(dt)
    else:
        s["q"], s["k"], s["v"] = (x.to(dt).transpose(1, 2).contiguous() for x in (q, k, v))      # [B, H, N, D]
    s["q_start"] = s["k_start"] = None
    if c["packed"]:
        sums = lambda x: _int32([sum(x[:i]) for i in range(b + 1)])  # noqa: E731
        s["q_start"] = sums(new)
        s["k_start"] = sums(rows) if n != m else s["q_start"]
    s["out"] = torch.zeros(s["q"].shape, dtype=dt, device="cuda")
    s["lse"] = torch.zeros((hq, n) if c["packed"] else (b, hq, n), device="cuda") if c["lse"] else None
    if own:
        from paper_2412_08521_amd import binding as B
        p = B.PromptParams(b, hq, h, d, n, m, dtype=B.EMS_F32 if c["f32"] else B.EMS_BF16)
        s["p"] = p
        s["ws"] = torch.empty(max(B.ems_prompt_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")


def _prepare_paged(c, s, u, gen):
    b, hq, h, d, ps, dt = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_size"], _dtype(c)
    new, rows = _geometry(c)
    pool, s["table"] = _pages(c, rows, gen)
    s["lens"] = _int32(rows)
    s["pos_pages"] = None
    if c.get("evicted"):
        gone = torch.rand((pool, h, ps), device="cuda", generator=gen) < c["evicted"]
        at = torch.randint(0, 1 << 20, (pool, h, ps), device="cuda", generator=gen, dtype=torch.int32)
        s["pos_pages"] = torch.where(gone, MASKED, at)
    k, v = _page_rows(c, pool, u, gen, True), _page_rows(c, pool, u, gen, False)
    if c["kind"] == "chunk":
        s["k_pages"], s["v_pages"] = k, v
        n = c["new"]
        # [B, N, Hq, D], as the projection leaves the queries
        s["q"] = _seeking(c, torch.randn((b, n, hq, d), device="cuda", generator=gen), u).to(dt).transpose(1, 2)
        s["new_len"] = _int32(new) if c["ragged"] else None
        s["out"] = torch.zeros((b, n, hq, d), dtype=dt, device="cuda").transpose(1, 2)
        s["lse"] = torch.zeros((b, hq, n), device="cuda") if c["lse"] else None
    else:
        step = max(1, (1 << 27) // (h * ps * d))
        for name, x in (("k", k), ("v", v)):
            s[name + "_pages"] = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
            s[name + "_scale"] = torch.empty(x.shape[:3], dtype=torch.uint8, device="cuda")
            for i in range(0, pool, step):
                s[name + "_pages"][i:i + step], s[name + "_scale"][i:i + step] = _quantized(x[i:i + step].float())
    if c["kind"] == "store8":
        n, nq = c["new"], hq if c["with_q"] else 0
        x = torch.randn((b, n, nq + 2 * h, d), device="cuda", generator=gen).to(dt)
        views = [x[:, :, i:j].transpose(1, 2) for i, j in ((0, nq), (nq, nq + h), (nq + h, nq + 2 * h))]
        s["q"], s["k"], s["v"] = (views[0] if nq else None), views[1], views[2]
        s["start"] = _int32([m - i for m, i in zip(rows, new)])
        s["new_len"] = _int32(new) if c["ragged"] else None
        # 10000^(-2i/rot), the usual frequencies
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().cuda() if c["rot"] else None
        s["q_out"] = torch.zeros((b, hq, n, d), dtype=dt, device="cuda") if nq else None
        s["len_out"] = torch.zeros(b, dtype=torch.int32, device="cuda")
        s["k_out"], s["v_out"] = (torch.zeros((b, h, max(rows), d), dtype=dt, device="cuda") for _ in range(2))
    if c["kind"] == "attend8":
        s["q"] = _seeking(c, torch.randn((b, hq, d), device="cuda", generator=gen), u).to(dt)
        s["out"] = torch.zeros((b, hq, d), dtype=dt, device="cuda")
        s["lse"] = torch.zeros((b, hq), device="cuda") if c["lse"] else None
    if own:
        from paper_2412_08521_amd import binding as B
        p = B.PagedParams(b, hq, h, d, ps, pool, s["table"].shape[1], dtype=B.EMS_F32 if c["f32"] else B.EMS_BF16)
        s["p"] = p
        if c["kind"] == "chunk":
            s["cache"] = B.PagedCache(p, s["k_pages"], s["v_pages"], s["table"], positions=s["pos_pages"])
            ws = B.ems_paged_chunk_workspace_bytes(p, c["new"])
        else:
            s["cache"] = B.QuantCache(p, s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"], positions=s["pos_pages"])
            ws = B.ems_quant_workspace_bytes(p)
        s["ws"] = torch.empty(max(ws, 256), dtype=torch.uint8, device="cuda")


# ---- one pass

def run(state):
    s = state
    c = s["case"]
    if own:
        return _run_own(c, s)
    return {"prompt": _plain_prompt, "chunk": _plain_chunk, "store8": _plain_store8, "attend8": _plain_attend8}[c["kind"]](c, s)


def _run_own(c, s):
    from paper_2412_08521_amd import binding as B
    if c["kind"] == "prompt":
        return B.ems_prompt_attention(s["p"], s["q"], s["k"], s["v"], q_start=s["q_start"], k_start=s["k_start"],
                                      want_lse=c["lse"], ws=s["ws"], out=(s["out"], s["lse"]))
    if c["kind"] == "chunk":
        return B.ems_paged_chunk_attention(s["p"], s["cache"], s["lens"], s["q"], new_len=s["new_len"], want_lse=c["lse"],
                                           ws=s["ws"], out=(s["out"], s["lse"]))
    if c["kind"] == "store8":
        q_out = B.ems_quant_append(s["p"], s["cache"], s["start"], s["k"], s["v"], new_len=s["new_len"],
                                    inv_freq=s["inv_freq"], interleaved=c["interleaved"], q=s["q"], q_out=s["q_out"],
                                    len_out=s["len_out"])
        k, v = B.ems_quant_read(s["p"], s["cache"], s["len_out"], out=(s["k_out"], s["v_out"]))
        return k, v, q_out, s["len_out"]
    return B.ems_quant_attention(s["p"], s["cache"], s["lens"], s["q"], want_lse=c["lse"], ws=s["ws"],
                                  out=(s["out"], s["lse"]))


def _softmax_rows(logits, live, v):
    """logits, live [..., G, L] and v [..., L, D], masked rows of v finite -> output and log-sum-exp; an empty row gives
    zeros and -inf."""
    logits = torch.where(live, logits, -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = (logits - top).exp()
    total = p.sum(dim=-1, keepdim=True)
    out = torch.where(total > 0, (p @ v) / total, 0.0)
    return out, (top + total.log())[..., 0]


def _attention(c, q, k, v, seen, live, most):
    """q [B, Hq, N, D], k, v [B, Hkv, M, D] in 32 bits, seen [B, N] rows that a query sees, live [B, Hkv, M] or None, most:
    the largest that any of the first i queries sees, by i -> out [B, Hq, N, D], lse [B, Hq, N], queries taken as many at a
    time as two gigabytes of scores hold."""
    b, hq, n, d = q.shape
    h, m = k.shape[1], k.shape[2]
    g = hq // h
    out, lse = torch.empty_like(q), torch.empty((b, hq, n), device="cuda")
    step = max(1, (1 << 29) // (b * hq * m))
    for i in range(0, n, step):
        j = min(n, i + step)
        w = most(j)
        logits = (q[:, :, i:j].reshape(b, h, g * (j - i), d) @ k[:, :, :w].transpose(-1, -2)) * d ** -0.5
        on = (torch.arange(w, device="cuda") < seen[:, i:j, None])[:, None, None]                    # [B, 1, 1, n, w]
        if live is not None:
            on = on & live[:, :, None, None, :w]
        o, z = _softmax_rows(logits.view(b, h, g, j - i, w), on, v[:, :, None, :w])
        out[:, :, i:j] = o.reshape(b, hq, j - i, d)
        lse[:, :, i:j] = z.reshape(b, hq, j - i)
    return out, lse


def _plain_prompt(c, s):
    new, rows = _geometry(c)
    n, m, d, dt = max(new), max(rows), c["head_dim"], _dtype(c)
    iq, ik = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    if not c["packed"]:
        seen = (iq + 1 + m - n).expand(c["batch"], n)
        out, lse = _attention(c, s["q"].float(), s["k"].float(), s["v"].float(), seen, None, lambda i: i + m - n)
        out = out.to(dt)
        return (out, lse) if c["lse"] else out
    q_len, k_len = s["q_start"].diff(), s["k_start"].diff()
    at = lambda start, i, most: (start[:-1, None] + i).clamp(max=most - 1).long()  # noqa: E731
    q, k, v = (x[at(start, i, len(x))].float().transpose(1, 2) for x, start, i in
               ((s["q"], s["q_start"], iq), (s["k"], s["k_start"], ik), (s["v"], s["k_start"], ik)))
    seen = torch.minimum(iq + 1 + (k_len - q_len)[:, None], k_len[:, None])
    out, lse = _attention(c, q, k, v, seen, None, lambda i: min(m, i + max(x - y for x, y in zip(rows, new))))
    on = iq < q_len[:, None]
    s["out"][:sum(new)] = out.transpose(1, 2)[on].to(dt)
    if not c["lse"]:
        return s["out"]
    s["lse"][:, :sum(new)] = lse.transpose(1, 2)[on].T
    return s["out"], s["lse"]


def _gathered(c, s, pages, b0, b1, width):
    """The pages' rows of sequences b0..b1, side by side: [b, Hkv, width, ...]."""
    x = pages[s["table"][b0:b1, :width // c["page_size"]].clamp(min=0).long()].transpose(1, 2)
    return x.reshape(x.shape[:2] + (width,) + tuple(pages.shape[3:]))


def _plain_chunk(c, s):
    new, rows = _geometry(c)
    b, n, h, d, ps = c["batch"], c["new"], c["kv_heads"], c["head_dim"], c["page_size"]
    q_len = s["new_len"] if s["new_len"] is not None else _int32([n] * b)
    i = torch.arange(n, device="cuda")
    width = s["table"].shape[1] * ps
    # as many sequences at a time as about two gigabytes of rows hold
    step = max(1, (1 << 29) // (h * width * d))
    for b0 in range(0, b, step):
        b1 = min(b, b0 + step)
        w = -(-max(rows[b0:b1]) // ps) * ps
        seen = torch.minimum(i + 1 + (s["lens"] - q_len)[b0:b1, None], s["lens"][b0:b1, None])
        live = _gathered(c, s, s["pos_pages"], b0, b1, w) >= 0 if s["pos_pages"] is not None else None
        k, v = (_gathered(c, s, s[x], b0, b1, w).float() for x in ("k_pages", "v_pages"))
        out, lse = _attention(c, s["q"][b0:b1].float(), k, v, seen, live, lambda j: w)
        on = (i < q_len[b0:b1, None])[:, None]
        s["out"][b0:b1] = torch.where(on[..., None], out.to(_dtype(c)), s["out"][b0:b1])
        if c["lse"]:
            s["lse"][b0:b1] = torch.where(on, lse, s["lse"][b0:b1])
    return (s["out"], s["lse"]) if c["lse"] else s["out"]


def _turned(x, cos, sin, rot, interleaved):
    """x [B, H, N, D] in 32 bits, cos and sin [B, 1, N, rot / 2]."""
    a, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a0, a1 = a[..., 0::2], a[..., 1::2]
        out = torch.stack((a0 * cos - a1 * sin, a1 * cos + a0 * sin), dim=-1).flatten(-2)
    else:
        a0, a1 = a[..., :rot // 2], a[..., rot // 2:]
        out = torch.cat((a0 * cos - a1 * sin, a1 * cos + a0 * sin), dim=-1)
    return torch.cat((out, rest), dim=-1)


def _plain_store8(c, s):
    b, n, ps, dt = c["batch"], c["new"], c["page_size"], _dtype(c)
    i = torch.arange(n, device="cuda", dtype=torch.int32)
    slot = s["start"][:, None] + i
    on = (i < (s["new_len"][:, None] if s["new_len"] is not None else n)).expand(b, n)
    k, q = s["k"].float(), s["q"]
    if c["rot"]:
        angle = slot[:, None, :, None].double() * s["inv_freq"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        k = _turned(k, cos, sin, c["rot"], c["interleaved"])
        q = q if q is None else _turned(q.float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    bi, ni = on.nonzero(as_tuple=True)
    page, at = s["table"][bi, (slot[bi, ni] // ps).long()].long(), (slot[bi, ni] % ps).long()
    codes = [_quantized(x.float()[bi, :, ni]) for x in (k, s["v"])]
    s["k_pages"][page, :, at], s["k_scale"][page, :, at] = codes[0]
    s["v_pages"][page, :, at], s["v_scale"][page, :, at] = codes[1]
    if q is not None:
        s["q_out"][bi, :, ni] = q[bi, :, ni]
    s["len_out"].copy_(s["start"] + on.sum(1, dtype=torch.int32))
    width, m = s["table"].shape[1] * ps, s["k_out"].shape[2]
    there = (torch.arange(m, device="cuda") < s["len_out"][:, None])[:, None, :, None]
    values = (_value(_gathered(c, s, s[x + "_pages"], 0, b, width), _gathered(c, s, s[x + "_scale"], 0, b, width))[:, :, :m]
              for x in "kv")
    k_all, v_all = (torch.where(there, x.to(dt), 0.0) for x in values)
    return k_all, v_all, s["q_out"], s["len_out"]


def _plain_attend8(c, s):
    b, hq, h, d, ps = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_size"]
    rows = _geometry(c)[1]
    out, lse = [], []
    step = max(1, (1 << 29) // (h * s["table"].shape[1] * ps * d))
    for b0 in range(0, b, step):
        b1 = min(b, b0 + step)
        w = -(-max(rows[b0:b1]) // ps) * ps
        k, v = (_value(_gathered(c, s, s[x + "_pages"], b0, b1, w), _gathered(c, s, s[x + "_scale"], b0, b1, w)) for x in "kv")
        live = _gathered(c, s, s["pos_pages"], b0, b1, w) >= 0 if s["pos_pages"] is not None else None
        o, z = _attention(c, s["q"][b0:b1, :, None].float(), k, v, s["lens"][b0:b1, None], live, lambda j: w)
        out.append(o[:, :, 0].to(_dtype(c)))
        lse.append(z[:, :, 0])
    out = torch.cat(out)
    return (out, torch.cat(lse)) if c["lse"] else out


# ---- the same in 64 bits, from the definitions

def exact(case, seed):
    """None in the place of lengths."""
    c = case
    s = prepare(c, seed)
    if c["kind"] == "store8":
        return _exact_store8(c, s)
    h, hq, d = c["kv_heads"], c["q_heads"], c["head_dim"]
    g = hq // h
    new, rows = _geometry(c)
    out = s["out"].double()
    lse = s["lse"].double() if s["lse"] is not None else None
    for i, (n, m) in enumerate(zip(new, rows)):
        n_q = n if c["kind"] != "attend8" else 1
        for j in range(h):
            keep = slice(None)
            if c["kind"] == "prompt":
                at, kat = sum(new[:i]), sum(rows[:i])
                k, v = (s[x][kat:kat + m, j] if c["packed"] else s[x][i, j] for x in "kv")
            else:
                pages = s["table"][i, :-(-m // c["page_size"])].long()
                k, v = (_rows_of(s, x, pages, j)[:m] for x in "kv")
                if s["pos_pages"] is not None:
                    keep = s["pos_pages"][pages, j].reshape(-1)[:m] >= 0
            k, v = k.double()[keep], v.double()[keep]
            number = torch.arange(m, device="cuda")[keep]
            for a in range(j * g, (j + 1) * g):
                for q0 in range(0, n_q, 4096):
                    q1 = min(n_q, q0 + 4096)
                    if c["kind"] == "prompt" and c["packed"]:
                        where = (slice(at + q0, at + q1), a)
                    elif c["kind"] == "attend8":
                        where = (i, slice(a, a + 1))
                    else:
                        where = (i, a, slice(q0, q1))
                    last = torch.arange(q0, q1, device="cuda")[:, None] + (m - n_q)
                    w = int((number <= q1 - 1 + m - n_q).sum())
                    x = s["q"][where].double() @ k[:w].T / math.sqrt(d)
                    x.masked_fill_(number[:w] > last, -math.inf)
                    z = torch.logsumexp(x, dim=1) if w else torch.full((q1 - q0,), -math.inf, dtype=torch.float64, device="cuda")
                    o = (x - torch.where(z > -math.inf, z, 0.0)[:, None]).exp_() @ v[:w]
                    out[where] = o
                    if lse is not None:
                        lse[(a, where[0]) if c["kind"] == "prompt" and c["packed"] else where] = z
    return (out, lse) if c["lse"] else out


def _rows_of(s, x, pages, j):
    """A sequence's rows of one head."""
    rows = s[x + "_pages"][pages, j].flatten(0, 1)
    if x + "_scale" not in s:
        return rows
    return rows.double() * torch.exp2(s[x + "_scale"][pages, j].flatten().double() - 127)[:, None]


def _exact_store8(c, s):
    h, hq, ps, rot, half = c["kv_heads"], c["q_heads"], c["page_size"], c["rot"], c["rot"] // 2
    new, rows = _geometry(c)
    k_all, v_all = s["k_out"].double(), s["v_out"].double()
    qo = s["q_out"].double() if s["q_out"] is not None else None
    # columns of the first and of the second element of every pair
    pair = torch.arange(half, device="cuda")
    one, two = (2 * pair, 2 * pair + 1) if c["interleaved"] else (pair, pair + half)
    for i, (n, m) in enumerate(zip(new, rows)):
        pos = torch.arange(m - n, m, device="cuda")
        pages = s["table"][i, :-(-m // ps)].long()
        for src, dst in (("k", k_all), ("v", v_all), ("q", qo)):
            if s[src] is None:
                continue
            x = s[src][i, :, :n].double()
            if rot and src != "v":
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, None].double() * s["inv_freq"].double())
                z = torch.complex(x[..., one], x[..., two]) * turn
                x[..., one], x[..., two] = z.real, z.imag
            if src == "q":
                dst[i, :, :n] = x
                continue
            for j in range(h):
                dst[i, j, :m - n] = _rows_of(s, src, pages, j)[:m - n]
            dst[i, :, m - n:m] = _nearest(x)
    return k_all, v_all, qo, None


def _nearest(x):
    """What rows of 64-bit numbers are in the cache: e4m3 numbers (steps of 2^-3 of the leading power of two, from 2^-6
    down 2^-9) times the row's power of two."""
    top = x.abs().amax(dim=-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-126))
    scale = torch.where(top > 448 * scale, 2 * scale, torch.where((top <= 224 * scale) & (scale > 2.0 ** -126), scale / 2, scale))
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))) / 8
    return torch.round(y / step) * step * scale
