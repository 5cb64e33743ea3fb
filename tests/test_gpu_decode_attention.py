"""GPU parity of the attention over the compact cache (ems_decode_attention) with a plain 64-bit form."""
import sys

import pytest
import torch

import ems_inputs
from gpu_util import dev_tensor
from paged_ref import assert_within, attention
from paper_2412_08521_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = B.EMS_BF16, B.EMS_F32


def _log(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _token(p, gen):
    return [torch.randn((p.batch, h, p.head_dim), generator=gen).to(p.torch_dtype) for h in (p.q_heads, p.kv_heads, p.kv_heads)]


def _check(p, st, q, k_new, v_new, out, lse):
    dt = p.torch_dtype
    scale = p.softmax_scale if p.softmax_scale > 0 else p.head_dim ** -0.5
    g = p.q_heads // p.kv_heads
    host = {x: getattr(st, x).cpu() for x in ("k_cache", "v_cache", "tok_row", "tok_norm", "row_norm")}
    for i in range(p.batch):
        for h in range(p.kv_heads):
            row = host["tok_row"][i, h].long()
            live = (row >= 0) & (row < p.budget)
            at = torch.where(live, row, 0)
            norm = host["row_norm"][i, h].double()[at]
            f = torch.where(norm > 0, host["tok_norm"][i, h].double() / norm, 0.0)
            k = torch.cat((host["k_cache"][i, h].double()[at] * f[:, None], k_new[i, h].double()[None]))
            v = torch.cat((host["v_cache"][i, h].double()[at], v_new[i, h].double()[None]))
            ref = attention(q[i, h * g:(h + 1) * g], k, v, torch.cat((live, torch.ones(1, dtype=torch.bool))), scale, dt)
            assert_within(out[i, h * g:(h + 1) * g], ref[0], ref[2], f"out of {i}, {h}")
            assert_within(lse[i, h * g:(h + 1) * g], ref[1], ref[3], f"lse of {i}, {h}")


def _made_up(b, hq, hkv, d, budget, window, ratio, mode, seed, scale=0.0):
    """A state with free elements, rows of norm 0 and rows that do not exist, in tables of every kind."""
    n = budget + int(ratio * budget) + 5
    p = B.EmsParams(b, hq, hkv, d, n, window, budget, merge_ratio=ratio, dtype=mode, softmax_scale=scale)
    gen = torch.Generator().manual_seed(seed)
    dt = p.torch_dtype
    kc, vc = (torch.randn((b, hkv, budget + 1, d), generator=gen).to(dt) for _ in range(2))
    n_imp, n_tbm = B.ems_partition_sizes(p)
    t = n_imp + n_tbm + window
    kc[:, :, 1] = 0
    norm = kc[:, :, :budget].float().norm(dim=-1)
    rows = torch.randint(-1, budget, (b, hkv, t), generator=gen, dtype=torch.int32)
    rows[torch.rand((b, hkv, t), generator=gen) < 0.2] = -1
    rows[:, 0, :2] = torch.tensor([1, budget], dtype=torch.int32)[:min(2, t)]
    st = B.DecodeState(p, kc.cuda(), vc.cuda())
    st.row_norm.copy_(norm)
    st.tok_row.copy_(rows)
    st.tok_norm.copy_(torch.rand((b, hkv, t), generator=gen) * 12)
    return p, st, gen


@pytest.mark.parametrize("mode", [BF16, F32])
@pytest.mark.parametrize("shape", [
    # (b, hq, hkv, d, budget, window, ratio): tables of up to 255 elements are one block's, longer ones shared
    (1, 1, 1, 64, 2, 1, 0.0),
    (2, 4, 2, 128, 40, 8, 0.5),
    (1, 8, 1, 64, 170, 16, 0.5),          # 255 elements and the new token fill one block's step
    (1, 8, 1, 64, 171, 16, 0.5),          # 256 and the new token
    (3, 6, 2, 128, 333, 33, 2.0),
    (2, 12, 4, 64, 1000, 32, 0.25),
    (1, 20, 1, 128, 2048, 64, 0.5),
    (5, 3, 3, 128, 63, 62, 0.0),
])
def test_decode_attention_matches_64_bits(shape, mode):
    _log("decode attention", shape, mode)
    p, st, gen = _made_up(*shape, mode, seed=shape[4], scale=0.2 if shape[4] == 40 else 0.0)
    q, k, v = _token(p, gen)
    dev = [x.cuda() for x in (q, k, v)]
    out, lse = B.ems_decode_attention(p, st, *dev, want_lse=True)
    assert torch.equal(out, B.ems_decode_attention(p, st, *dev))
    _check(p, st, q, k, v, out, lse)


@pytest.mark.parametrize("mode", [BF16, F32])
def test_decode_attention_of_an_empty_table_is_the_new_value(mode):
    p, st, gen = _made_up(2, 4, 2, 64, 300, 16, 0.5, mode, seed=1)
    st.tok_row.fill_(-1)
    st.v_cache.fill_(float("nan"))
    st.k_cache.fill_(float("inf"))
    q, k, v = _token(p, gen)
    out, lse = B.ems_decode_attention(p, st, q.cuda(), k.cuda(), v.cuda(), want_lse=True)
    assert torch.equal(out.cpu(), v.repeat_interleave(2, 1))
    x = (q.double() * k.double().repeat_interleave(2, 1)).sum(-1) * 0.125
    bound = (q.double() * k.double().repeat_interleave(2, 1)).abs().sum(-1) * 0.125 * 70 * 2.0 ** -24 + 8 * 2.0 ** -24 * x.abs() + 2.0 ** -22
    assert_within(lse, x, bound, "lse")


@pytest.mark.parametrize("mode", [BF16, F32])
def test_decode_attention_of_queries_off_a_boundary(mode):
    p, st, gen = _made_up(2, 4, 2, 128, 700, 16, 0.5, mode, seed=3)
    q, k, v = _token(p, gen)
    flat = torch.zeros(q.numel() + 1, dtype=q.dtype).cuda()
    flat[1:] = q.flatten().cuda()
    off = flat[1:].view(q.shape)
    assert off.data_ptr() % 16
    out = B.ems_decode_attention(p, st, off, k.cuda(), v.cuda())
    assert torch.equal(out, B.ems_decode_attention(p, st, q.cuda(), k.cuda(), v.cuda()))
    with pytest.raises(B.EmsError, match="invalid argument"):
        B.ems_decode_attention(p, st, off, off[:, :2].contiguous(), off.flatten()[:v.numel()].view(v.shape))


@pytest.mark.parametrize("mode", [BF16, F32])
def test_generation_over_the_compact_cache(mode):
    """Prompt to generation: attention, then the step that changes the state, token after token; the output agrees with
    64 bits, and with the weights of the step itself."""
    b, hq, hkv, d, n, w, nb = 2, 8, 2, 128, 900, 16, 150
    p = B.EmsParams(b, hq, hkv, d, n, w, nb, merge_ratio=1.5, tau=0.3, pool_kernel=3, dtype=mode)
    inp = ems_inputs.small(b, hq, hkv, d, n, seed=4)
    q, k, v = (dev_tensor(getattr(inp, x), mode) for x in "qkv")
    s_glo, s_loc = B.ems_global_local_score(p, q, k)
    imp, tbm = B.ems_select(p, s_glo, s_loc)
    st = B.ems_decode_init(p, B.ems_evict_merge(p, k, v, imp, tbm), tbm, s_glo, s_loc)
    gen = torch.Generator().manual_seed(8)
    for t in range(w + 3):
        qn, kn, vn = _token(p, gen)
        dev = [x.cuda() for x in (qn, kn, vn)]
        out, lse = B.ems_decode_attention(p, st, *dev, want_lse=True)
        _check(p, st, qn, kn, vn, out, lse)
        rows = torch.where(st.tok_row >= 0, st.tok_row, 0).long()
        values = torch.cat((st.v_cache.gather(2, rows[..., None].expand(*rows.shape, d)), dev[2][:, :, None]), 2).double()
        attn = B.ems_decode_step(p, st, t, *dev, want_attn=True)["attn"].double().view(b, hkv, hq // hkv, -1)
        mixed = (attn @ values).view(b, hq, d)
        # the step's weights are within 2e-5 of 64 bits (its own test).  The output's: |q||k| scale is about 11, so twice
        # 11 * 132 half steps of float32, 2^-16 for the pieces, 2 * 400 half steps for the sums: 2.5e-4 in all
        bound = (attn @ values.abs()).view(b, hq, d) * 3e-4 + mixed.abs() * torch.finfo(p.torch_dtype).eps / 2 * 1.02
        assert_within(out, mixed.cpu(), bound.cpu(), f"token {t}")


def test_decode_attention_replays_from_a_graph():
    p, st, gen = _made_up(3, 8, 2, 128, 600, 16, 0.5, BF16, seed=2)
    buf = [x.cuda() for x in _token(p, gen)]
    ws = torch.empty(B.ems_decode_attention_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    outs = [(torch.empty_like(buf[0]), torch.empty(buf[0].shape[:2], device="cuda")) for _ in range(2)]
    B.ems_decode_attention(p, st, *buf, want_lse=True, ws=ws, out=outs[0])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.ems_decode_attention(p, st, *buf, want_lse=True, ws=ws, out=outs[1])
    torch.cuda.synchronize()
    for _ in range(4):
        for x, y in zip(buf, _token(p, gen)):
            x.copy_(y)
        B.ems_decode_attention(p, st, *buf, want_lse=True, ws=ws, out=outs[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
