"""Tensors that take another's place in a cache or a decode state: a call sees them, and refuses what does not fit, before
anything runs.  Without a GPU: host tensors pass for those of the current device."""
import pytest
import torch

from paper_2412_08521_amd import binding as B


@pytest.fixture
def host_device(monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: -1)


def _state(p):
    n_imp, n_tbm = B.ems_partition_sizes(p)
    t, i32, f32 = n_imp + n_tbm + p.window, torch.int32, torch.float32
    st = object.__new__(B.DecodeState)
    rows = (p.batch, p.kv_heads, p.budget + 1, p.head_dim)
    st.k_cache, st.v_cache = torch.zeros(rows, dtype=p.torch_dtype), torch.zeros(rows, dtype=p.torch_dtype)
    heads = (p.batch, p.kv_heads)
    for name, n, dtype in (("row_norm", p.budget, f32), ("entry_count", n_imp, i32), ("entry_tok", n_imp, i32), ("tok_pos", t, i32),
                           ("tok_row", t, i32), ("tok_norm", t, f32), ("tok_glo", t, f32), ("tok_past", t, f32), ("tok_cur", t, f32)):
        setattr(st, name, torch.zeros(heads + (n,), dtype=dtype))
    st.step_count = torch.zeros(1, dtype=i32)
    return st


def test_decode_state_refuses_replaced_tensors():
    """Every tensor of a state keeps its shape and type, so the calls need not look at all of them."""
    p = B.EmsParams(2, 4, 2, 64, 400, 16, 100, merge_ratio=0.5)
    st = _state(p)
    for name in B.STATE_FIELDS:
        x = getattr(st, name)
        strided = x.repeat_interleave(2, -1)[..., ::2]
        for other in (torch.cat((x, x)), x.double(), x[None]) + (() if strided.is_contiguous() else (strided,)):
            with pytest.raises(ValueError, match=name):
                setattr(st, name, other)
        assert getattr(st, name) is x


def test_decode_attention_refuses_a_state_of_other_parameters(host_device):
    p = B.EmsParams(2, 4, 2, 64, 400, 16, 100, merge_ratio=0.5)
    q, k, v = (torch.zeros((2, h, 64), dtype=torch.bfloat16) for h in (4, 2, 2))
    for kw, name in ((dict(budget=101), "k_cache"), (dict(merge_ratio=0.6), "tok_row"), (dict(merge_ratio=0.4), "tok_row")):
        with pytest.raises(ValueError, match=name):
            B.ems_decode_attention(B.EmsParams(**{**dict(batch=2, q_heads=4, kv_heads=2, head_dim=64, seq_len=400, window=16, budget=100,
                                                         merge_ratio=0.5), **kw}), _state(p), q, k, v)


def test_decode_state_takes_a_replaced_tensors_address():
    p = B.EmsParams(2, 4, 2, 64, 400, 16, 100, merge_ratio=0.5)
    st = _state(p)
    first = st.c()
    assert st.c() is first
    for name in B.STATE_FIELDS:
        new = getattr(st, name).clone()
        setattr(st, name, new)
        assert getattr(st.c(), name) == new.data_ptr()


def test_paged_cache_refuses_replaced_tensors(host_device):
    p = B.PagedParams(2, 4, 2, 64, 16, 10, 5)
    rows = (10, 2, 16, 64)

    def cache():
        return B.PagedCache(p, torch.zeros(rows, dtype=torch.bfloat16), torch.zeros(rows, dtype=torch.bfloat16),
                            torch.zeros((2, 5), dtype=torch.int32), positions=torch.zeros(rows[:3], dtype=torch.int32))
    wide = torch.zeros((2, 9), dtype=torch.int32)
    for name, x in (("page_table", wide[:, :5]), ("page_table", torch.zeros((2, 5), dtype=torch.int64)), ("k_pages", torch.zeros(rows)), ("v_pages", torch.zeros(rows, dtype=torch.float16)),
                    ("v_pages", torch.zeros((10, 2, 64, 16), dtype=torch.bfloat16).transpose(2, 3)),
                    ("positions", torch.zeros(rows[:3])), ("positions", torch.zeros((10, 2, 32), dtype=torch.int32)[..., ::2])):
        with pytest.raises(ValueError, match=name):
            setattr(cache(), name, x)
    c = cache()
    c.device_index = 0                                        # had its tensors been the first device's
    for name in ("k_pages", "v_pages", "page_table", "positions"):
        with pytest.raises(ValueError, match=f"{name} must be a tensor of the current device"):
            setattr(c, name, getattr(c, name).clone())
    # of its kind, but of another size: the call refuses it
    for name, x in (("v_pages", torch.zeros((9,) + rows[1:], dtype=torch.bfloat16)), ("positions", torch.zeros((10, 2, 8), dtype=torch.int32)),
                    ("page_table", wide), ("k_pages", torch.zeros((11,) + rows[1:], dtype=torch.bfloat16))):
        c = cache()
        setattr(c, name, x)
        with pytest.raises(ValueError, match="does not fit"):
            c._c(p, -1)
    # a longer table with parameters of its width, and no positions any more
    c = cache()
    c.page_table, c.positions = wide, None
    got = c._c(B.PagedParams(2, 4, 2, 64, 16, 10, 9), -1)._obj
    assert got.page_table == wide.data_ptr() and got.positions is None


def test_tensors_that_are_let_go(host_device):
    """None frees a tensor's memory; a call has nothing to run on then, old addresses least of all."""
    p = B.EmsParams(2, 4, 2, 64, 400, 16, 100, merge_ratio=0.5)
    st = _state(p)
    st.c()
    st.v_cache = None
    with pytest.raises(AttributeError):
        st.c()
    with pytest.raises(ValueError, match="v_cache"):
        st.v_cache = st.k_cache[:1].clone()
    st.v_cache = st.k_cache.clone()
    assert st.c().v_cache == st.v_cache.data_ptr()
    pp = B.PagedParams(2, 4, 2, 64, 16, 10, 5)
    rows = [torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16) for _ in range(2)]
    cache = B.PagedCache(pp, *rows, torch.zeros((2, 5), dtype=torch.int32))
    cache.k_pages = None
    with pytest.raises(AttributeError):
        cache._c(pp, -1)
    with pytest.raises(ValueError, match="k_pages"):
        cache.k_pages = rows[0].float()
    cache.k_pages = rows[0]
    assert cache._c(pp, -1)._obj.k_pages == rows[0].data_ptr()
