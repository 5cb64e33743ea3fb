"""Host-side checks of the paged cache's calls and of the attention over the compact cache, without a GPU: sizes, and the
refusal of what no kernel could run."""
import ctypes as C

import pytest
import torch

from paged_ref import attention, rotated
from paper_2412_08521_amd import binding as B

INVALID, UNSUPPORTED, WORKSPACE = B.EMS_ERR_INVALID_ARG, B.EMS_ERR_UNSUPPORTED, B.EMS_ERR_WORKSPACE
D = 1 << 12                                       # an address that no refused call touches


def _paged(**kw):
    return B.PagedParams(**{**dict(batch=2, q_heads=4, kv_heads=2, head_dim=128, page_size=16, num_pages=100, max_pages=50), **kw})


def _append(p, **kw):
    """The status of a call whose arguments are all there, but for `kw`."""
    st = lambda: B.ems_strides(1024, 128, 512)  # noqa: E731
    a = dict(cache=B.ems_paged_cache(D, D, None, D), n_new=1, start=D, new_len=None, k=D, ks=st(), v=D, vs=st(), pos=None,
             ps=None, freq=D, rot=128, inter=0, q=D, qs=st(), q_out=D, qos=st(), len_out=None)
    a.update(kw)
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return B.lib().ems_paged_append(ref(p and p.c()), ref(a["cache"]), a["n_new"], a["start"], a["new_len"], a["k"], ref(a["ks"]),
                                    a["v"], ref(a["vs"]), a["pos"], ref(a["ps"]), a["freq"], a["rot"], a["inter"], a["q"],
                                    ref(a["qs"]), a["q_out"], ref(a["qos"]), a["len_out"], None)


def _attend(p, **kw):
    a = dict(cache=B.ems_paged_cache(D, D, None, D), lens=D, q=D, qs=B.ems_strides(512, 128, 0), out=D, lse=None, ws=D, n=1 << 40)
    a.update(kw)
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return B.lib().ems_paged_attention(ref(p and p.c()), ref(a["cache"]), a["lens"], a["q"], ref(a["qs"]), a["out"], a["lse"],
                                       a["ws"], a["n"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), INVALID), (dict(q_heads=5), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
    (dict(page_size=0), INVALID), (dict(num_pages=0), INVALID), (dict(max_pages=-1), INVALID), (dict(dtype=2), INVALID),
    (dict(softmax_scale=float("nan")), INVALID), (dict(softmax_scale=float("inf")), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(num_pages=1 << 26), UNSUPPORTED), (dict(max_pages=(1 << 26) + 1), UNSUPPORTED),
    (dict(batch=1 << 23), UNSUPPORTED), (dict(q_heads=65538), UNSUPPORTED),
    (dict(batch=1 << 20, max_pages=1 << 20), UNSUPPORTED)])
def test_paged_parameters(kw, code):
    p = _paged(**kw)
    assert _append(p) == code and _attend(p) == code
    with pytest.raises(B.EmsError) as e:
        B.ems_paged_workspace_bytes(p)
    assert e.value.status == code


def test_append_arguments():
    p = _paged()
    s = B.ems_strides(1024, 128, 512)
    for kw in (dict(cache=None), dict(cache=B.ems_paged_cache(None, D, None, D)), dict(cache=B.ems_paged_cache(D, None, None, D)),
               dict(cache=B.ems_paged_cache(D, D, None, None)), dict(cache=B.ems_paged_cache(D + 8, D, None, D)),
               dict(cache=B.ems_paged_cache(D, D + 2, None, D)), dict(n_new=0), dict(n_new=-1), dict(start=None), dict(k=None),
               dict(ks=None), dict(v=None), dict(vs=None), dict(pos=D), dict(freq=None), dict(rot=0), dict(rot=-16), dict(rot=144),
               dict(q=None), dict(q_out=None), dict(qs=None), dict(qos=None), dict(len_out=D), dict(len_out=D + 4), dict(len_out=D - 4),
               dict(start=D + 64, new_len=D, len_out=D + 4)):
        assert _append(p, **kw) == INVALID, kw
    assert _append(None) == INVALID
    assert _append(p, rot=24) == UNSUPPORTED and _append(p, rot=2) == UNSUPPORTED
    assert _append(p, n_new=1 << 30) == UNSUPPORTED
    assert _append(p, pos=D, ps=s, rot=8) == UNSUPPORTED


def test_attention_arguments():
    p = _paged()
    need = B.ems_paged_workspace_bytes(p)
    assert need > 0 and need % 256 == 0
    for kw in (dict(cache=None), dict(cache=B.ems_paged_cache(D, D, None, None)), dict(cache=B.ems_paged_cache(D, D + 8, None, D)),
               dict(lens=None), dict(q=None), dict(qs=None), dict(out=None), dict(out=D + 8)):
        assert _attend(p, **kw) == INVALID, kw
    assert _attend(None) == INVALID
    for kw in (dict(ws=None), dict(ws=D + 16), dict(n=need - 1)):
        assert _attend(p, **kw) == WORKSPACE, kw


def test_which_calls_share_sequences_between_blocks():
    """A workspace is needed where they do: sequences over 256 KB of keys and values, over 1 MB where the blocks of whole
    sequences are 256 or more."""
    def shared(rows, **kw):
        return B.ems_paged_workspace_bytes(_paged(page_size=1, max_pages=rows, **kw)) > 0
    assert not shared(512) and shared(513)                                               # 512 bytes a row
    assert not shared(1024, head_dim=64) and shared(1025, head_dim=64)
    assert not shared(512, head_dim=64, dtype=B.EMS_F32) and shared(513, head_dim=64, dtype=B.EMS_F32)
    for more in (dict(batch=128), dict(batch=32, q_heads=8, kv_heads=8), dict(batch=64, q_heads=66)):    # the last: two blocks' q-heads
        assert not shared(2048, **more) and shared(2049, **more)
    assert shared(2048, batch=127)
    p = lambda budget, ratio, n=1 << 16: B.EmsParams(1, 4, 2, 64, n, 16, budget, merge_ratio=ratio)  # noqa: E731
    need = B.ems_decode_attention_workspace_bytes
    assert need(p(682, 0.5)) == 0 and need(p(683, 0.5)) > 0                              # 1023 and 1024 elements and the new token


def test_decode_attention_arguments():
    lib = B.lib()
    p = B.EmsParams(1, 6, 2, 64, 4096, 16, 1000, merge_ratio=0.5)
    cp = p.c()
    need = B.ems_decode_attention_workspace_bytes(p)
    assert need > 0

    def call(cp=cp, st=None, q=D, k=D, v=D, out=D, ws=D, n=1 << 40, **null):
        st = B.ems_decode_state(*[null.get(x, D) for x in B.STATE_FIELDS])
        return lib.ems_decode_attention(C.byref(cp), C.byref(st), q, k, v, out, None, ws, n, None)

    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(k=D + 2), dict(v=D + 8), dict(out=D + 2),
               dict(k_cache=None), dict(v_cache=None), dict(k_cache=D + 8), dict(row_norm=None), dict(tok_row=None),
               dict(tok_norm=None), dict(cp=B.EmsParams(1, 6, 2, 64, 4096, 16, 16).c())):
        assert call(**kw) == INVALID, kw
    assert call(cp=B.EmsParams(1, 6, 2, 80, 4096, 16, 1000).c()) == UNSUPPORTED
    assert call(cp=B.EmsParams(1, 65536, 2, 64, 4096, 16, 1000).c()) == UNSUPPORTED
    for kw in (dict(ws=None), dict(ws=D + 16), dict(n=need - 1)):
        assert call(**kw) == WORKSPACE, kw
    assert lib.ems_decode_attention(C.byref(cp), None, D, D, D, D, None, D, 1 << 40, None) == INVALID
    assert lib.ems_decode_attention(None, None, D, D, D, D, None, D, 1 << 40, None) == INVALID
    assert lib.ems_decode_attention_workspace_bytes(C.byref(B.EmsParams(1, 6, 2, 64, 4096, 16, 16).c()), None) == INVALID


def test_binding_refuses_host_tensors_and_other_shapes():
    p = _paged()
    rows = (100, 2, 16, 128)
    k = torch.zeros(rows, dtype=torch.bfloat16)
    table = torch.zeros((2, 50), dtype=torch.int32)
    with pytest.raises(ValueError, match="k_pages must be a tensor of the current device"):
        B.PagedCache(p, k, k, table)
    with pytest.raises(ValueError, match="current device"):
        B.alloc_paged_cache(p, table)
    cache = object.__new__(B.PagedCache)                      # a cache, had its tensors been a device's
    cache.k_pages, cache.v_pages, cache.page_table, cache.positions = k, k, table, None
    lens = torch.zeros(2, dtype=torch.int32)
    q, kn = torch.zeros((2, 4, 128), dtype=torch.bfloat16), torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    cache.device_index = 77
    for call in (lambda: B.ems_paged_attention(p, cache, lens, q), lambda: B.ems_paged_append(p, cache, lens, kn, kn)):
        with pytest.raises(ValueError, match="the cache must be on the current device"):
            call()
    cache.device_index = B._current_device()
    with pytest.raises(ValueError, match="q must be a tensor of the current device"):
        B.ems_paged_attention(p, cache, lens, q)
    with pytest.raises(ValueError, match="k must be a tensor of the current device"):
        B.ems_paged_append(p, cache, lens, kn, kn)
    for kw in (dict(num_pages=101), dict(page_size=32), dict(max_pages=51), dict(batch=1), dict(dtype=B.EMS_F32),
               dict(kv_heads=4), dict(head_dim=64)):
        with pytest.raises(ValueError, match="does not fit"):
            cache._c(_paged(**kw), cache.device_index)


# ---- the plain forms themselves

def test_plain_rotation_turns_pairs_and_keeps_norms():
    x = torch.randn((3, 5, 64), generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    pos = torch.arange(15).view(3, 5) * 1000
    freq = torch.tensor([1.0, 0.5, 0.25, 0.0] * 4)
    for inter in (False, True):
        y, _ = rotated(x, pos, freq, inter)
        assert torch.equal(y[..., 32:], x[..., 32:])
        assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1), rtol=1e-13)
        back, _ = rotated(y, -pos, freq, inter)
        assert torch.allclose(back, x, atol=1e-12)
        same = 3 if inter else None                           # frequency 0 turns nothing
        assert torch.equal(y[..., 2 * 3] if same else y[..., 3], x[..., 2 * 3] if same else x[..., 3])
    # scores depend on the distance alone
    a, b = x[0, 0], x[0, 1]
    dots = [rotated(a, torch.tensor(7 + s), freq, True)[0] @ rotated(b, torch.tensor(3 + s), freq, True)[0] for s in (0, 90)]
    assert abs(dots[0] - dots[1]) < 1e-11


def test_plain_attention_against_torch():
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 16), (40, 16), (40, 16)))
    live = torch.rand(40, generator=gen) < 0.6
    out, lse, _, _ = attention(q, k, v, live, 0.25, torch.float32)
    w = torch.softmax((q @ k.T * 0.25).masked_fill(~live, -torch.inf), 1)
    assert torch.allclose(out, w @ v, atol=1e-13) and lse.shape == (3,)
    none = attention(q, k, v, torch.zeros(40, dtype=torch.bool), 0.25, torch.float32)
    assert not none[0].any() and (none[1] == -torch.inf).all()
