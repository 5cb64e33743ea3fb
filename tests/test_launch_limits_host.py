"""Sizes past what a launch may have (2^32 threads) are refused on the host, like others that no kernel could run."""
import pytest

from paper_2412_08521_amd import binding as B
from test_paged_host import UNSUPPORTED, _append, _attend


def _one(**kw):
    return B.PagedParams(**{**dict(batch=1, q_heads=1, kv_heads=1, head_dim=128, page_size=1, num_pages=1, max_pages=1), **kw})


def test_most_sequences_of_an_attention():
    p = _one(batch=1 << 24)
    assert _attend(p) == UNSUPPORTED
    with pytest.raises(B.EmsError) as e:
        B.ems_paged_workspace_bytes(p)
    assert e.value.status == UNSUPPORTED
    assert B.ems_paged_workspace_bytes(_one(batch=(1 << 24) - 1)) == 0
    with pytest.raises(B.EmsError) as e:
        B.ems_decode_attention_workspace_bytes(B.EmsParams(1 << 24, 1, 1, 64, 8, 1, 2))
    assert e.value.status == UNSUPPORTED


@pytest.mark.parametrize("d,dtype,most", [(128, B.EMS_F32, 16), (128, B.EMS_BF16, 32), (64, B.EMS_F32, 32)])
def test_most_tokens_of_an_append(d, dtype, most):
    """By 16 or 32 tokens a block (64 for rows of 128 bytes, whose limit the number of rows reaches first)."""
    p = _one(head_dim=d, dtype=dtype)
    past = ((1 << 24) - 1) * most + 1
    assert past * 3 < 1 << 31                                # not refused for its rows
    assert _append(p, n_new=past, rot=d, q=None, q_out=None) == UNSUPPORTED
