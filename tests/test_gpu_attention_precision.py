"""The attention of one new token keeps its weights in 32 bits: outputs that show their last digits, and the rms of the
error where roundings are many (tests/test_attention_precision.py shows what these checks find)."""
import sys

import pytest
import torch

from paged_ref import assert_within, gather
from paper_2412_08521_amd import binding as B
from precision_ref import Rms, cancelling, cancelling_bound, rms_parts
from test_gpu_paged import _attend_case

pytestmark = pytest.mark.gpu

MODES = [B.EMS_BF16, B.EMS_F32]


def _log(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _cases(group, d, count, dtype):
    got = [cancelling(group, d, seed, dtype) for seed in range(count)]
    return [torch.stack(x) for x in list(zip(*got))[:3]] + [got[0][3]]


def _hold(out, q, dtype):
    for i in range(len(q)):
        ref, bound = cancelling_bound(q[i], dtype)
        assert_within(out[i].diagonal(), ref, bound, f"sequence {i}")


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("columns", [1, 200, 20000])          # whole sequences, shared ones, ones read past the caches
@pytest.mark.parametrize("group,d", [(1, 64), (16, 64), (16, 128), (20, 64), (40, 128)])
def test_paged_weights_keep_32_bits(group, d, columns, masked, mode):
    _log("paged weights", group, d, columns, masked, mode)
    b, ps = 6, 8
    p = B.PagedParams(b, group, 1, d, ps, b, columns, softmax_scale=1.0, dtype=mode)
    q, k, v, _ = _cases(group, d, b, p.torch_dtype)
    table = torch.full((b, columns), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(b - 1, -1, -1)
    cache = B.alloc_paged_cache(p, table.cuda(), positions=masked)
    lens = torch.zeros(b, dtype=torch.int32).cuda()
    B.ems_paged_append(p, cache, torch.zeros_like(lens), k[:, None].cuda(), v[:, None].cuda(), len_out=lens)
    _hold(B.ems_paged_attention(p, cache, lens, q.cuda()), q, p.torch_dtype)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("budget", [3, 1100])                  # whole sequences, shared ones
@pytest.mark.parametrize("group,d", [(16, 64), (16, 128), (20, 64), (40, 128)])
def test_compact_weights_keep_32_bits(group, d, budget, mode):
    _log("compact weights", group, d, budget, mode)
    b = 6
    p = B.EmsParams(b, group, 1, d, budget + 4, 1, budget, softmax_scale=1.0, merge_ratio=0.0, dtype=mode)
    q, k, v, _ = _cases(group, d, b, p.torch_dtype)
    kc, vc = (torch.zeros((b, 1, budget + 1, d), dtype=p.torch_dtype) for _ in range(2))
    vc[:, 0, 0], vc[:, 0, budget - 1] = v[:, 0], v[:, 1]      # keys 0 of norm 0; the third row is the new token's
    st = B.DecodeState(p, kc.cuda(), vc.cuda())
    st.tok_row[:, :, 0], st.tok_row[:, :, -1] = budget - 1, 0
    _hold(B.ems_decode_attention(p, st, q.cuda(), k[:, 2:].cuda(), v[:, 2:].cuda()), q, p.torch_dtype)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("masked", [None, 0.4])
@pytest.mark.parametrize("shape,columns", [
    ((3, 8, 2, 128, 16, [256, 255, 65]), None),
    ((2, 6, 6, 64, 16, [200, 33]), None),
    ((2, 12, 3, 128, 16, [3000, 511]), None),
    ((3, 21, 3, 64, 24, [1500, 1, 777]), None),
    ((2, 40, 2, 64, 5, [1200, 40]), 40000),
    ((2, 40, 2, 128, 16, [2100, 600]), 8000),
])
def test_rms_of_the_error(shape, columns, masked, mode):
    _log("rms", shape, columns, masked, mode)
    p, cache, lens, q, out = _attend_case(*shape, mode, masked=masked, columns=columns, seed=17)
    host = [x.cpu() for x in (cache.k_pages, cache.v_pages, cache.page_table, q, out)]
    pos = cache.positions.cpu() if masked is not None else torch.zeros(cache.k_pages.shape[:3])
    rms, g = Rms(p.torch_dtype), p.q_heads // p.kv_heads
    for i, n in enumerate(lens.tolist()):
        for h in range(p.kv_heads):
            k, v = (gather(x, host[2][i], h, n) for x in host[:2])
            heads = slice(h * g, (h + 1) * g)
            rms.add(host[4][i, heads], *rms_parts(host[3][i, heads], k, v, gather(pos, host[2][i], h, n) >= 0, p.head_dim ** -0.5))
    assert rms.ratio() < 3, rms.ratio()
