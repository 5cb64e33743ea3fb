"""Table elements of a compact cache that name no row are free, whatever number they hold (ems_decode_attention)."""
import sys

import pytest
import torch

from paper_2412_08521_amd import binding as B
from test_gpu_decode_attention import _check, _made_up, _token

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [B.EMS_BF16, B.EMS_F32])
@pytest.mark.parametrize("free", [-2, -3, -(1 << 31), 0, 1, (1 << 31) - 1])           # from 0 on: so many past the last row
@pytest.mark.parametrize("shape", [
    (2, 4, 2, 128, 40, 8, 0.5),
    (1, 8, 1, 64, 171, 16, 0.5),
    (2, 12, 4, 64, 1000, 32, 0.25),       # shared between blocks
    (1, 20, 1, 128, 2048, 64, 0.5),
])
def test_elements_without_a_row(shape, free, mode):
    print("[case]", shape, free, mode, file=sys.stderr, flush=True)
    p, st, gen = _made_up(*shape, mode, seed=shape[4])
    st.tok_row[st.tok_row >= p.budget] = -1
    none = st.tok_row < 0
    assert none.any() and not none.all()
    q, k, v = _token(p, gen)
    dev = [x.cuda() for x in (q, k, v)]
    want = B.ems_decode_attention(p, st, *dev, want_lse=True)
    number = free if free < 0 else min(p.budget + free, (1 << 31) - 1)
    st.tok_row[none] = number
    st.tok_norm[none] = float("nan")
    out, lse = B.ems_decode_attention(p, st, *dev, want_lse=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    st.tok_norm[none] = 1.0
    _check(p, st, q, k, v, out, lse)
    st.tok_row.fill_(number)                                   # nothing but the new token
    out = B.ems_decode_attention(p, st, *dev)
    assert torch.equal(out.cpu(), v.repeat_interleave(p.q_heads // p.kv_heads, 1))
