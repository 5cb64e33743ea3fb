"""Thin ctypes binding of libems_hip.so (C ABI in include/ems.h).

Argument marshalling only: every step of the path runs in the HIP kernels.  PyTorch is used
for device memory and the current stream.  There is no CPU fallback: if the library is not
built, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libems_hip.so")

EMS_OK = 0
EMS_ERR_INVALID_ARG = -1
EMS_ERR_UNSUPPORTED = -2
EMS_ERR_WORKSPACE = -3
EMS_ERR_LAUNCH = -4
EMS_BF16 = 0
EMS_F32 = 1
EMS_SIM_KEY = 0
EMS_SIM_VALUE = 1
EMS_SIM_KEY_VALUE = 2
EMS_STEP_FROM_STATE = -1

EXPORTS = ("ems_version", "ems_strerror", "ems_partition_sizes", "ems_workspace_bytes",
           "ems_global_local_score", "ems_attention_lse", "ems_global_local_score_from_lse",
           "ems_select", "ems_evict_merge", "ems_evict_merge_variant", "ems_evict_merge_static", "ems_expand",
           "ems_decode_workspace_bytes", "ems_decode_init", "ems_decode_step",
           "ems_sparsity_rate", "ems_redundancy_rate",
           "ems_decode_attention_workspace_bytes", "ems_decode_attention",
           "ems_paged_workspace_bytes", "ems_paged_append", "ems_paged_attention",
           "ems_paged_chunk_workspace_bytes", "ems_paged_chunk_attention",
           "ems_prompt_workspace_bytes", "ems_prompt_attention",
           "ems_quant_append", "ems_quant_read", "ems_quant_workspace_bytes", "ems_quant_attention")


class ems_params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("seq_len", C.c_int32), ("window", C.c_int32),
                ("budget", C.c_int32), ("merge_ratio", C.c_float), ("tau", C.c_float),
                ("pool_kernel", C.c_int32), ("softmax_scale", C.c_float), ("dtype", C.c_int32)]


STATE_FIELDS = ("k_cache", "v_cache", "row_norm", "entry_count", "entry_tok", "tok_pos", "tok_row",
                "tok_norm", "tok_glo", "tok_past", "tok_cur", "step_count")


class ems_decode_state(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in STATE_FIELDS]


class ems_paged_params(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("batch", "q_heads", "kv_heads", "head_dim", "page_size", "num_pages",
                                               "max_pages")] + [("softmax_scale", C.c_float), ("dtype", C.c_int32)]


class ems_paged_cache(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("k_pages", "v_pages", "positions", "page_table")]


class ems_quant_cache(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("k_pages", "v_pages", "k_scale", "v_scale", "positions", "page_table")]


class ems_prompt_params(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("batch", "q_heads", "kv_heads", "head_dim", "q_rows", "k_rows")] + [
        ("softmax_scale", C.c_float), ("dtype", C.c_int32)]


class ems_strides(C.Structure):
    _fields_ = [(name, C.c_int64) for name in ("batch", "head", "token")]


class EmsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


@dataclass
class EmsParams:
    batch: int
    q_heads: int
    kv_heads: int
    head_dim: int
    seq_len: int
    window: int
    budget: int = 0
    merge_ratio: float = 0.5
    tau: float = 0.6
    pool_kernel: int = 7
    softmax_scale: float = 0.0
    dtype: int = EMS_BF16

    def c(self) -> ems_params:
        return ems_params(self.batch, self.q_heads, self.kv_heads, self.head_dim, self.seq_len,
                          self.window, self.budget, self.merge_ratio, self.tau,
                          self.pool_kernel, self.softmax_scale, self.dtype)

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == EMS_F32 else torch.bfloat16


@dataclass(frozen=True)
class PagedParams:
    batch: int
    q_heads: int
    kv_heads: int
    head_dim: int
    page_size: int
    num_pages: int
    max_pages: int
    softmax_scale: float = 0.0
    dtype: int = EMS_BF16

    def __post_init__(self):                       # what every call needs of them, made once (they do not change)
        put = lambda name, x: object.__setattr__(self, name, x)  # noqa: E731
        put("_c", ems_paged_params(self.batch, self.q_heads, self.kv_heads, self.head_dim, self.page_size, self.num_pages,
                                   self.max_pages, self.softmax_scale, self.dtype))
        put("torch_dtype", torch.float32 if self.dtype == EMS_F32 else torch.bfloat16)
        put("_q_row", (self.batch, self.q_heads, self.head_dim))
        put("_pages", (self.num_pages, self.kv_heads, self.page_size, self.head_dim))
        put("_positions", self._pages[:3])
        put("_table", (self.batch, self.max_pages))

    def c(self) -> ems_paged_params:
        return self._c


@dataclass(frozen=True)
class PromptParams:
    """q_rows, k_rows: of every sequence, or of all of them together where they are packed."""
    batch: int
    q_heads: int
    kv_heads: int
    head_dim: int
    q_rows: int
    k_rows: int
    softmax_scale: float = 0.0
    dtype: int = EMS_BF16

    def __post_init__(self):                       # made once, as those of PagedParams
        put = lambda name, x: object.__setattr__(self, name, x)  # noqa: E731
        put("_c", ems_prompt_params(self.batch, self.q_heads, self.kv_heads, self.head_dim, self.q_rows, self.k_rows,
                                    self.softmax_scale, self.dtype))
        put("torch_dtype", torch.float32 if self.dtype == EMS_F32 else torch.bfloat16)

    def c(self) -> ems_prompt_params:
        return self._c


_lib = None


def lib():
    """Load the built library (never builds, never falls back)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built: run `python -m paper_2412_08521_amd.build`")
        l = C.CDLL(LIB_PATH)
        l.ems_version.restype = C.c_int
        l.ems_strerror.restype = C.c_char_p
        l.ems_strerror.argtypes = [C.c_int]
        P = C.POINTER(ems_params)
        l.ems_partition_sizes.argtypes = [P, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        l.ems_workspace_bytes.argtypes = [P] + [C.POINTER(C.c_size_t)] * 3
        l.ems_global_local_score.argtypes = [P] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
        l.ems_attention_lse.argtypes = [P] + [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
        l.ems_global_local_score_from_lse.argtypes = [P] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
        l.ems_select.argtypes = [P] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
        l.ems_evict_merge.argtypes = [P] + [C.c_void_p] * 12 + [C.c_size_t, C.c_void_p]
        l.ems_evict_merge_variant.argtypes = ([P, C.c_int] + [C.c_void_p] * 13 + [C.c_size_t, C.c_void_p])
        l.ems_evict_merge_static.argtypes = [P] + [C.c_void_p] * 12
        l.ems_expand.argtypes = [P] + [C.c_void_p] * 10
        l.ems_sparsity_rate.argtypes = [P, C.c_float] + [C.c_void_p] * 5
        l.ems_redundancy_rate.argtypes = [P] + [C.c_void_p] * 5
        S = C.POINTER(ems_decode_state)
        l.ems_decode_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        l.ems_decode_init.argtypes = [P] + [C.c_void_p] * 7 + [S, C.c_void_p]
        l.ems_decode_step.argtypes = [P, S, C.c_int32] + [C.c_void_p] * 6 + [C.c_void_p, C.c_size_t, C.c_void_p]
        l.ems_decode_attention_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t)]
        l.ems_decode_attention.argtypes = [P, S] + [C.c_void_p] * 6 + [C.c_size_t, C.c_void_p]
        PP, PC, ST = C.POINTER(ems_paged_params), C.POINTER(ems_paged_cache), C.POINTER(ems_strides)
        l.ems_paged_workspace_bytes.argtypes = [PP, C.POINTER(C.c_size_t)]
        l.ems_paged_append.argtypes = ([PP, PC, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, ST, C.c_void_p, ST,
                                        C.c_void_p, ST, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, ST, C.c_void_p, ST,
                                        C.c_void_p, C.c_void_p])
        l.ems_paged_attention.argtypes = [PP, PC, C.c_void_p, C.c_void_p, ST] + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p]
        PP8, PR = C.POINTER(ems_quant_cache), C.POINTER(ems_prompt_params)
        l.ems_paged_chunk_workspace_bytes.argtypes = [PP, C.c_int32, C.POINTER(C.c_size_t)]
        l.ems_paged_chunk_attention.argtypes = ([PP, PC, C.c_int32] + [C.c_void_p] * 3 + [ST, C.c_void_p, ST] + [C.c_void_p] * 2 +
                                                [C.c_size_t, C.c_void_p])
        l.ems_prompt_workspace_bytes.argtypes = [PR, C.POINTER(C.c_size_t)]
        l.ems_prompt_attention.argtypes = [PR] + [C.c_void_p, ST] * 3 + [C.c_void_p] * 3 + [ST] + [C.c_void_p] * 2 + [C.c_size_t, C.c_void_p]
        l.ems_quant_append.argtypes = [PP, PP8] + l.ems_paged_append.argtypes[2:]
        l.ems_quant_read.argtypes = [PP, PP8, C.c_int32, C.c_void_p, C.c_void_p, ST, C.c_void_p, ST, C.c_void_p]
        l.ems_quant_workspace_bytes.argtypes = [PP, C.POINTER(C.c_size_t)]
        l.ems_quant_attention.argtypes = [PP, PP8] + l.ems_paged_attention.argtypes[2:]
        for name in EXPORTS[2:]:
            getattr(l, name).restype = C.c_int
        _lib = l
    return _lib


def strerror(status: int) -> str:
    return lib().ems_strerror(int(status)).decode()


def ems_version() -> int:
    return int(lib().ems_version())


def ems_partition_sizes(p: EmsParams):
    return _partition_sizes(p.c())


def _partition_sizes(cp: ems_params):
    a, b = C.c_int32(0), C.c_int32(0)
    rc = lib().ems_partition_sizes(C.byref(cp), C.byref(a), C.byref(b))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_partition_sizes")
    return a.value, b.value


def ems_workspace_bytes(p: EmsParams, full: bool = True):
    return _workspace_bytes(p.c(), full)


def _workspace_bytes(cp: ems_params, full: bool):
    s, t, u = C.c_size_t(0), C.c_size_t(0), C.c_size_t(0)
    rc = lib().ems_workspace_bytes(C.byref(cp), C.byref(s), C.byref(t) if full else None,
                                   C.byref(u) if full else None)
    if rc != EMS_OK:
        raise EmsError(rc, "ems_workspace_bytes")
    return int(s.value), int(t.value), int(u.value)


# A call on a short prompt, or a generated token, costs the host more than its kernels run for: the helpers
# below do one thing each, addresses go to ctypes as plain numbers (the argument types are declared), and
# every entry point builds the parameter structure once and asks for workspace sizes only where it
# allocates (one layer's compression of 1024 tokens: 83 -> 62 us of host time).
def _ptr(t):
    return None if t is None else t.data_ptr()


# torch's own short way to the current stream's handle, where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _check_tensor(t, shape, dtype, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _workspace(cp: ems_params, which: int, device, ws=None):
    """The caller's workspace, or a new one: which = 0 score, 1 select, 2 evict-merge."""
    if ws is None:
        ws = torch.empty(max(_workspace_bytes(cp, which > 0)[which], 256), dtype=torch.uint8, device=device)
    return ws


def ems_global_local_score(p: EmsParams, q, k, want_lse: bool = False, ws=None, out=None):
    """-> (s_glo, s_loc[, lse]) device f32 tensors [B,Hkv,N] ([B,Hq,N])."""
    _check_tensor(q, (p.batch, p.q_heads, p.seq_len, p.head_dim), p.torch_dtype, "q")
    _check_tensor(k, (p.batch, p.kv_heads, p.seq_len, p.head_dim), p.torch_dtype, "k")
    dev, cp = q.device, p.c()
    ws = _workspace(cp, 0, dev, ws)
    if out is None:
        s_glo = torch.empty((p.batch, p.kv_heads, p.seq_len), dtype=torch.float32, device=dev)
        s_loc = torch.empty_like(s_glo)
    else:
        s_glo, s_loc = out
    lse = torch.empty((p.batch, p.q_heads, p.seq_len), dtype=torch.float32, device=dev) if want_lse else None
    rc = lib().ems_global_local_score(C.byref(cp), _ptr(q), _ptr(k), _ptr(s_glo), _ptr(s_loc),
                                      _ptr(lse), _ptr(ws), ws.numel(), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_global_local_score")
    return (s_glo, s_loc, lse) if want_lse else (s_glo, s_loc)


def ems_attention_lse(p: EmsParams, q, k, ws=None, out=None):
    """-> lse device f32 [B,Hq,N] (natural log)."""
    _check_tensor(q, (p.batch, p.q_heads, p.seq_len, p.head_dim), p.torch_dtype, "q")
    _check_tensor(k, (p.batch, p.kv_heads, p.seq_len, p.head_dim), p.torch_dtype, "k")
    cp = p.c()
    ws = _workspace(cp, 0, q.device, ws)
    lse = out if out is not None else torch.empty((p.batch, p.q_heads, p.seq_len),
                                                  dtype=torch.float32, device=q.device)
    rc = lib().ems_attention_lse(C.byref(cp), _ptr(q), _ptr(k), _ptr(lse), _ptr(ws), ws.numel(),
                                 _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_attention_lse")
    return lse


def ems_global_local_score_from_lse(p: EmsParams, q, k, lse, ws=None, out=None):
    """-> (s_glo, s_loc) from a caller-supplied natural-log row log-sum-exp."""
    _check_tensor(q, (p.batch, p.q_heads, p.seq_len, p.head_dim), p.torch_dtype, "q")
    _check_tensor(k, (p.batch, p.kv_heads, p.seq_len, p.head_dim), p.torch_dtype, "k")
    _check_tensor(lse, (p.batch, p.q_heads, p.seq_len), torch.float32, "lse")
    dev, cp = q.device, p.c()
    ws = _workspace(cp, 0, dev, ws)
    if out is None:
        s_glo = torch.empty((p.batch, p.kv_heads, p.seq_len), dtype=torch.float32, device=dev)
        s_loc = torch.empty_like(s_glo)
    else:
        s_glo, s_loc = out
    rc = lib().ems_global_local_score_from_lse(C.byref(cp), _ptr(q), _ptr(k), _ptr(lse),
                                               _ptr(s_glo), _ptr(s_loc), _ptr(ws), ws.numel(),
                                               _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_global_local_score_from_lse")
    return s_glo, s_loc


def ems_select(p: EmsParams, s_glo, s_loc, want_pooled: bool = False, ws=None, out=None):
    """-> (imp_idx, tbm_idx[, pooled]) device tensors."""
    shape = (p.batch, p.kv_heads, p.seq_len)
    _check_tensor(s_glo, shape, torch.float32, "s_glo")
    _check_tensor(s_loc, shape, torch.float32, "s_loc")
    dev, cp = s_glo.device, p.c()
    n_imp, n_tbm = _partition_sizes(cp)
    ws = _workspace(cp, 1, dev, ws)
    if out is None:
        imp = torch.empty((p.batch, p.kv_heads, n_imp), dtype=torch.int32, device=dev)
        tbm = torch.empty((p.batch, p.kv_heads, n_tbm), dtype=torch.int32, device=dev)
    else:
        imp, tbm = out
    pooled = torch.empty(shape, dtype=torch.float32, device=dev) if want_pooled else None
    rc = lib().ems_select(C.byref(cp), _ptr(s_glo), _ptr(s_loc), _ptr(pooled), _ptr(imp),
                          _ptr(tbm) if n_tbm else None, _ptr(ws), ws.numel(), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_select")
    return (imp, tbm, pooled) if want_pooled else (imp, tbm)


def alloc_evict_merge_outputs(p: EmsParams, device):
    n_imp, n_tbm = ems_partition_sizes(p)
    B, H, D, Nb = p.batch, p.kv_heads, p.head_dim, p.budget
    i32, f32 = torch.int32, torch.float32
    return dict(
        k_out=torch.empty((B, H, Nb + 1, D), dtype=p.torch_dtype, device=device),
        v_out=torch.empty((B, H, Nb + 1, D), dtype=p.torch_dtype, device=device),
        kept_pos=torch.empty((B, H, Nb), dtype=i32, device=device),
        tbm_dest=torch.empty((B, H, n_tbm), dtype=i32, device=device),
        tbm_sim=torch.empty((B, H, n_tbm), dtype=f32, device=device),
        k_norm=torch.empty((B, H, n_imp + n_tbm), dtype=f32, device=device),
        slot_count=torch.empty((B, H, n_imp + 1), dtype=i32, device=device),
    )


def ems_evict_merge(p: EmsParams, k, v, imp_idx, tbm_idx, ws=None, out=None):
    """-> dict(k_out, v_out, kept_pos, tbm_dest, tbm_sim, k_norm, slot_count)."""
    shape = (p.batch, p.kv_heads, p.seq_len, p.head_dim)
    _check_tensor(k, shape, p.torch_dtype, "k")
    _check_tensor(v, shape, p.torch_dtype, "v")
    cp = p.c()
    n_imp, n_tbm = _partition_sizes(cp)
    _check_tensor(imp_idx, (p.batch, p.kv_heads, n_imp), torch.int32, "imp_idx")
    _check_tensor(tbm_idx, (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_idx")
    dev = k.device
    ws = _workspace(cp, 2, dev, ws)
    o = out if out is not None else alloc_evict_merge_outputs(p, dev)
    has = n_tbm > 0
    rc = lib().ems_evict_merge(C.byref(cp), _ptr(k), _ptr(v), _ptr(imp_idx),
                               _ptr(tbm_idx) if has else None, _ptr(o["k_out"]), _ptr(o["v_out"]),
                               _ptr(o["kept_pos"]), _ptr(o["tbm_dest"]) if has else None,
                               _ptr(o["tbm_sim"]) if has else None, _ptr(o["k_norm"]),
                               _ptr(o["slot_count"]), _ptr(ws), ws.numel(), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_evict_merge")
    return o


def ems_evict_merge_static(p: EmsParams, k, v, imp_idx, tbm_idx, out=None, k_norm: bool = True):
    """ems_evict_merge on the library's fixed scratch array: no workspace, nothing allocated by the
    call (pass `out` from alloc_evict_merge_outputs to keep the binding from allocating as well).
    With k_norm=False no key norms are returned and they live in the scratch array."""
    shape = (p.batch, p.kv_heads, p.seq_len, p.head_dim)
    _check_tensor(k, shape, p.torch_dtype, "k")
    _check_tensor(v, shape, p.torch_dtype, "v")
    cp = p.c()
    n_imp, n_tbm = _partition_sizes(cp)
    _check_tensor(imp_idx, (p.batch, p.kv_heads, n_imp), torch.int32, "imp_idx")
    _check_tensor(tbm_idx, (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_idx")
    o = dict(out) if out is not None else alloc_evict_merge_outputs(p, k.device)
    if not k_norm:
        o["k_norm"] = None
    has = n_tbm > 0
    rc = lib().ems_evict_merge_static(C.byref(cp), _ptr(k), _ptr(v), _ptr(imp_idx),
                                      _ptr(tbm_idx) if has else None, _ptr(o["k_out"]), _ptr(o["v_out"]),
                                      _ptr(o["kept_pos"]), _ptr(o["tbm_dest"]) if has else None,
                                      _ptr(o["tbm_sim"]) if has else None, _ptr(o["k_norm"]),
                                      _ptr(o["slot_count"]), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_evict_merge_static")
    return o


def ems_evict_merge_variant(p: EmsParams, similarity: int, k, v, token_weight, imp_idx, tbm_idx,
                            ws=None, out=None):
    """ems_evict_merge with the redundancy of `similarity` (EMS_SIM_*) and, when `token_weight`
    ([B, Hkv, N] f32) is given, the score-weighted merge.  Same outputs."""
    shape = (p.batch, p.kv_heads, p.seq_len, p.head_dim)
    _check_tensor(k, shape, p.torch_dtype, "k")
    _check_tensor(v, shape, p.torch_dtype, "v")
    if token_weight is not None:
        _check_tensor(token_weight, shape[:3], torch.float32, "token_weight")
    cp = p.c()
    n_imp, n_tbm = _partition_sizes(cp)
    _check_tensor(imp_idx, (p.batch, p.kv_heads, n_imp), torch.int32, "imp_idx")
    _check_tensor(tbm_idx, (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_idx")
    dev = k.device
    ws = _workspace(cp, 2, dev, ws)
    o = out if out is not None else alloc_evict_merge_outputs(p, dev)
    has = n_tbm > 0
    rc = lib().ems_evict_merge_variant(
        C.byref(cp), int(similarity), _ptr(k), _ptr(v), _ptr(token_weight), _ptr(imp_idx),
        _ptr(tbm_idx) if has else None, _ptr(o["k_out"]), _ptr(o["v_out"]), _ptr(o["kept_pos"]),
        _ptr(o["tbm_dest"]) if has else None, _ptr(o["tbm_sim"]) if has else None,
        _ptr(o["k_norm"]), _ptr(o["slot_count"]), _ptr(ws), ws.numel(), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_evict_merge_variant")
    return o


def ems_expand(p: EmsParams, merged: dict, tbm_idx, out=None):
    """Expand the compact cache `merged` (the dict ems_evict_merge returned) back to one
    key / value per kept token -> (k_exp, v_exp, pos_exp)."""
    cp = p.c()
    n_imp, n_tbm = _partition_sizes(cp)
    n_exp = n_imp + n_tbm + p.window
    dev = merged["k_out"].device
    _check_tensor(merged["k_out"], (p.batch, p.kv_heads, p.budget + 1, p.head_dim), p.torch_dtype, "k_cache")
    _check_tensor(merged["v_out"], (p.batch, p.kv_heads, p.budget + 1, p.head_dim), p.torch_dtype, "v_cache")
    _check_tensor(merged["kept_pos"], (p.batch, p.kv_heads, p.budget), torch.int32, "kept_pos")
    _check_tensor(merged["k_norm"], (p.batch, p.kv_heads, n_imp + n_tbm), torch.float32, "k_norm")
    _check_tensor(merged["tbm_dest"], (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_dest")
    _check_tensor(tbm_idx, (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_idx")
    if out is None:
        k_exp = torch.empty((p.batch, p.kv_heads, n_exp, p.head_dim), dtype=p.torch_dtype, device=dev)
        v_exp = torch.empty_like(k_exp)
        pos = torch.empty((p.batch, p.kv_heads, n_exp), dtype=torch.int32, device=dev)
    else:
        k_exp, v_exp, pos = out
    has = n_tbm > 0
    rc = lib().ems_expand(C.byref(cp), _ptr(merged["k_out"]), _ptr(merged["v_out"]),
                          _ptr(merged["kept_pos"]), _ptr(tbm_idx) if has else None,
                          _ptr(merged["tbm_dest"]) if has else None, _ptr(merged["k_norm"]),
                          _ptr(k_exp), _ptr(v_exp), _ptr(pos), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_expand")
    return k_exp, v_exp, pos


def ems_decode_workspace_bytes(p: EmsParams) -> int:
    n = C.c_size_t(0)
    cp = p.c()
    rc = lib().ems_decode_workspace_bytes(C.byref(cp), C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_decode_workspace_bytes")
    return int(n.value)


class DecodeState:
    """Device tensors of the decode-time state (see ems_decode_state in include/ems.h)."""

    def __init__(self, p: EmsParams, k_cache, v_cache):
        n_imp, n_tbm = ems_partition_sizes(p)
        B, H, Nb = p.batch, p.kv_heads, p.budget
        T = n_imp + n_tbm + p.window
        dev = k_cache.device
        _check_tensor(k_cache, (B, H, Nb + 1, p.head_dim), p.torch_dtype, "k_cache")
        _check_tensor(v_cache, (B, H, Nb + 1, p.head_dim), p.torch_dtype, "v_cache")
        self.n_tokens = T
        self.k_cache, self.v_cache = k_cache, v_cache
        # one slab for the nine small arrays: they are all touched by every step, and sitting in
        # one allocation keeps them on as few pages as possible
        shapes = [("row_norm", (B, H, Nb), torch.float32), ("entry_count", (B, H, n_imp), torch.int32),
                  ("entry_tok", (B, H, n_imp), torch.int32), ("tok_pos", (B, H, T), torch.int32),
                  ("tok_row", (B, H, T), torch.int32), ("tok_norm", (B, H, T), torch.float32),
                  ("tok_glo", (B, H, T), torch.float32), ("tok_past", (B, H, T), torch.float32),
                  ("tok_cur", (B, H, T), torch.float32), ("step_count", (1,), torch.int32)]
        sizes = [(4 * int(torch.Size(shape).numel()) + 255) // 256 * 256 for _, shape, _ in shapes]
        self.slab = torch.zeros(sum(sizes), dtype=torch.uint8, device=dev)
        off = 0
        for (name, shape, dtype), size in zip(shapes, sizes):
            n = int(torch.Size(shape).numel())
            setattr(self, name, self.slab[off:off + 4 * n].view(dtype).view(shape))
            off += size
        self.tok_pos.fill_(-1)
        self.tok_row.fill_(-1)

    def __setattr__(self, name, x):
        if name in STATE_FIELDS and x is not None:           # a tensor in another's place has to be like the first one there
            like = self.__dict__.setdefault("_like", {})
            if name in like:
                _check_dense(x, *like[name], name)
            else:
                like[name] = (x.get_device(), x.dtype, x.shape)
        self.__dict__[name] = x
        if name in STATE_FIELDS:
            self.__dict__["_c"] = None                       # its address is taken anew

    def c(self) -> ems_decode_state:
        if getattr(self, "_c", None) is None:                # made once: the tensors do not move
            self._c = ems_decode_state(*[getattr(self, name).data_ptr() for name in STATE_FIELDS])
        return self._c


def ems_decode_init(p: EmsParams, merged: dict, tbm_idx, s_glo, s_loc, state=None) -> DecodeState:
    """State for the generation from ems_evict_merge's outputs (`merged`; its k_out / v_out
    become the live cache and are updated in place by ems_decode_step)."""
    n_imp, n_tbm = ems_partition_sizes(p)
    shape = (p.batch, p.kv_heads, p.seq_len)
    _check_tensor(s_glo, shape, torch.float32, "s_glo")
    _check_tensor(s_loc, shape, torch.float32, "s_loc")
    _check_tensor(merged["kept_pos"], (p.batch, p.kv_heads, p.budget), torch.int32, "kept_pos")
    _check_tensor(merged["k_norm"], (p.batch, p.kv_heads, n_imp + n_tbm), torch.float32, "k_norm")
    _check_tensor(merged["tbm_dest"], (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_dest")
    _check_tensor(merged["slot_count"], (p.batch, p.kv_heads, n_imp + 1), torch.int32, "slot_count")
    _check_tensor(tbm_idx, (p.batch, p.kv_heads, n_tbm), torch.int32, "tbm_idx")
    st = state if state is not None else DecodeState(p, merged["k_out"], merged["v_out"])
    has = n_tbm > 0
    cp, cs = p.c(), st.c()
    rc = lib().ems_decode_init(C.byref(cp), _ptr(s_glo), _ptr(s_loc), _ptr(merged["kept_pos"]),
                               _ptr(tbm_idx) if has else None, _ptr(merged["tbm_dest"]) if has else None,
                               _ptr(merged["k_norm"]), _ptr(merged["slot_count"]), C.byref(cs), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_decode_init")
    return st


def ems_decode_step(p: EmsParams, st: DecodeState, step: int, q_new, k_new, v_new, want_attn=False,
                    ws=None, out=None):
    """One generated token -> dict(decision [B,Hkv,2], sim [B,Hkv], attn [B,Hq,T+1] or None)."""
    _check_tensor(q_new, (p.batch, p.q_heads, p.head_dim), p.torch_dtype, "q_new")
    _check_tensor(k_new, (p.batch, p.kv_heads, p.head_dim), p.torch_dtype, "k_new")
    _check_tensor(v_new, (p.batch, p.kv_heads, p.head_dim), p.torch_dtype, "v_new")
    dev = q_new.device
    if ws is None:
        ws = torch.empty(max(ems_decode_workspace_bytes(p), 256), dtype=torch.uint8, device=dev)
    if out is None:
        out = dict(decision=torch.empty((p.batch, p.kv_heads, 2), dtype=torch.int32, device=dev),
                   sim=torch.empty((p.batch, p.kv_heads), dtype=torch.float32, device=dev),
                   attn=torch.empty((p.batch, p.q_heads, st.n_tokens + 1), dtype=torch.float32, device=dev)
                   if want_attn else None)
    cp, cs = p.c(), st.c()
    rc = lib().ems_decode_step(C.byref(cp), C.byref(cs), int(step), _ptr(q_new), _ptr(k_new), _ptr(v_new),
                               _ptr(out.get("attn")), _ptr(out["decision"]), _ptr(out["sim"]),
                               _ptr(ws), ws.numel(), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_decode_step")
    return out


def ems_sparsity_rate(p: EmsParams, zeta: float, s_glo, s_loc):
    """Eq. 3 -> (rate [B,Hkv] f32, n_k [B,Hkv] i32)."""
    shape = (p.batch, p.kv_heads, p.seq_len)
    _check_tensor(s_glo, shape, torch.float32, "s_glo")
    _check_tensor(s_loc, shape, torch.float32, "s_loc")
    rate = torch.empty(shape[:2], dtype=torch.float32, device=s_glo.device)
    n_k = torch.empty(shape[:2], dtype=torch.int32, device=s_glo.device)
    cp = p.c()
    rc = lib().ems_sparsity_rate(C.byref(cp), float(zeta), _ptr(s_glo), _ptr(s_loc), _ptr(rate), _ptr(n_k),
                                 _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_sparsity_rate")
    return rate, n_k


def ems_redundancy_rate(p: EmsParams, k, v):
    """Eq. 4 -> (rate [B,Hkv] f32, best [B,Hkv,N] f32)."""
    shape = (p.batch, p.kv_heads, p.seq_len, p.head_dim)
    _check_tensor(k, shape, p.torch_dtype, "k")
    _check_tensor(v, shape, p.torch_dtype, "v")
    rate = torch.empty(shape[:2], dtype=torch.float32, device=k.device)
    best = torch.empty(shape[:3], dtype=torch.float32, device=k.device)
    cp = p.c()
    rc = lib().ems_redundancy_rate(C.byref(cp), _ptr(k), _ptr(v), _ptr(rate), _ptr(best), _stream())
    if rc != EMS_OK:
        raise EmsError(rc, "ems_redundancy_rate")
    return rate, best


# The calls of a generation's step are short: like the others they cost the host more than the device, and checks are
# most of what a call does here.  The current device is asked for once a call, by torch's short way to it, and a tensor is
# checked in one expression (append with queries: 10.2 -> 9.5 us a call).
def _refuse(t, dev, dtype, shape, name):
    if t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor of the current device")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _check_dense(t, dev, dtype, shape, name):
    """A contiguous device tensor of the current device (the launch goes to it)."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        _refuse(t, dev, dtype, shape, name)


_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_device():
    try:
        return _get_device() if _get_device is not None else torch.cuda.current_device()
    except (RuntimeError, AssertionError):            # no device: every tensor is refused
        return None


def _stream_of(dev):
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream


def _check_ws(ws, dev, need, p):
    if ws is None:
        return torch.empty(max(need(p), 256), dtype=torch.uint8, device="cuda")
    if ws.get_device() != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws: contiguous bytes of the current device")
    return ws


@functools.lru_cache(maxsize=512)
def _table_length(seq_len, window, budget, merge_ratio):
    """Tokens of a decode state's table; it depends on nothing else of the parameters."""
    return sum(_partition_sizes(EmsParams(1, 1, 1, 64, seq_len, window, budget, merge_ratio).c())) + window


@functools.lru_cache(maxsize=512)
def _strides(batch, head, token):
    return C.byref(ems_strides(batch, head, token))


def ems_decode_attention_workspace_bytes(p: EmsParams) -> int:
    n = C.c_size_t(0)
    cp = p.c()
    rc = lib().ems_decode_attention_workspace_bytes(C.byref(cp), C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_decode_attention_workspace_bytes")
    return int(n.value)


def ems_decode_attention(p: EmsParams, st: DecodeState, q_new, k_new, v_new, want_lse=False, ws=None, out=None):
    """Attention of one new token over the compact cache and itself -> out [B,Hq,D] (or (out, lse [B,Hq] f32) with
    want_lse).  Call it before the token's ems_decode_step.  `out`: (out, lse or None) to write to."""
    dev, dt, cp = _current_device(), p.torch_dtype, p.c()
    heads, shape = (p.batch, p.q_heads), (p.batch, p.kv_heads, p.head_dim)
    _check_dense(q_new, dev, dt, heads + shape[2:], "q_new")
    _check_dense(k_new, dev, dt, shape, "k_new")
    _check_dense(v_new, dev, dt, shape, "v_new")
    table = (p.batch, p.kv_heads, _table_length(p.seq_len, p.window, p.budget, p.merge_ratio))
    _check_dense(st.k_cache, dev, dt, (p.batch, p.kv_heads, p.budget + 1, p.head_dim), "k_cache")
    _check_dense(st.tok_row, dev, torch.int32, table, "tok_row")        # (the state's other tensors go with these two)
    ws = _check_ws(ws, dev, ems_decode_attention_workspace_bytes, p)
    o, lse = _attention_out(out, dev, want_lse, heads + shape[2:], dt)
    cs = st.c()
    rc = lib().ems_decode_attention(C.byref(cp), C.byref(cs), q_new.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
                                    o.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(), _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_decode_attention")
    return (o, lse) if want_lse else o


def _attention_out(out, dev, want_lse, shape, dtype):
    if out is None:
        return (torch.empty(shape, dtype=dtype, device="cuda"),
                torch.empty(shape[:2], dtype=torch.float32, device="cuda") if want_lse else None)
    o, lse = out
    _check_dense(o, dev, dtype, shape, "out")
    if not want_lse:
        return o, None
    if lse is None:
        raise ValueError("out: a tensor for the log-sum-exp is wanted")
    _check_dense(lse, dev, torch.float32, shape[:2], "lse")
    return o, lse


class PagedCache:
    """Device tensors of a paged cache (see ems_paged_cache in include/ems.h): k_pages, v_pages
    [num_pages, Hkv, page_size, D], page_table [B, max_pages] int32, and with `positions` [num_pages, Hkv, page_size]
    int32 the position of every row, negative = masked."""
    _dtypes = dict(k_pages=None, v_pages=None, page_table=torch.int32, positions=torch.int32)      # None: that of the parameters

    def __init__(self, p: PagedParams, k_pages, v_pages, page_table, positions=None):
        dev, dt = _current_device(), self._dtypes["k_pages"] or p.torch_dtype
        _check_dense(k_pages, dev, dt, p._pages, "k_pages")
        _check_dense(v_pages, dev, dt, p._pages, "v_pages")
        _check_dense(page_table, dev, torch.int32, p._table, "page_table")
        if positions is not None:
            _check_dense(positions, dev, torch.int32, p._positions, "positions")
        self.k_pages, self.v_pages, self.page_table, self.positions = k_pages, v_pages, page_table, positions
        self.device_index, self.dtype = dev, p.torch_dtype

    def __setattr__(self, name, t):
        # a tensor in another's place (a longer table, a larger pool) is checked here, its shape by the next call
        if t is not None and name in self.__dict__ and name in self._dtypes:
            _check_dense(t, self.device_index, self._dtypes[name] or self.dtype, t.shape, name)
        self.__dict__[name] = t

    def _c(self, p: PagedParams, dev):
        """The cache for a call on device `dev` with parameters that have to be those of its tensors."""
        k, pos = self.k_pages, self.positions
        if (k.shape != p._pages or self.v_pages.shape != p._pages or self.page_table.shape != p._table or k.dtype != p.torch_dtype or
                (pos is not None and pos.shape != p._positions)):
            raise ValueError(f"a cache of {tuple(k.shape)} rows with a table of {tuple(self.page_table.shape)} does not fit {p}")
        if self.device_index != dev:
            raise ValueError("the cache must be on the current device")
        return C.byref(ems_paged_cache(k.data_ptr(), self.v_pages.data_ptr(), _ptr(pos), self.page_table.data_ptr()))


class QuantCache(PagedCache):
    """Device tensors of a paged cache in 8 bits (see ems_quant_cache in include/ems.h): k_pages, v_pages
    [num_pages, Hkv, page_size, D] float8_e4m3fn, k_scale, v_scale [num_pages, Hkv, page_size] uint8 (s + 127 of a row's
    2^s), page_table and positions as in a PagedCache."""
    _dtypes = dict(PagedCache._dtypes, k_pages=torch.float8_e4m3fn, v_pages=torch.float8_e4m3fn, k_scale=torch.uint8,
                   v_scale=torch.uint8)

    def __init__(self, p: PagedParams, k_pages, v_pages, k_scale, v_scale, page_table, positions=None):
        dev = _current_device()
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _check_dense(t, dev, torch.uint8, p._positions, name)
        self.k_scale, self.v_scale = k_scale, v_scale
        super().__init__(p, k_pages, v_pages, page_table, positions)

    def _c(self, p: PagedParams, dev):
        k, pos = self.k_pages, self.positions
        if (k.shape != p._pages or self.v_pages.shape != p._pages or self.page_table.shape != p._table or
                self.k_scale.shape != p._positions or self.v_scale.shape != p._positions or
                (pos is not None and pos.shape != p._positions)):
            raise ValueError(f"a cache of {tuple(k.shape)} rows with a table of {tuple(self.page_table.shape)} does not fit {p}")
        if self.device_index != dev:
            raise ValueError("the cache must be on the current device")
        return C.byref(ems_quant_cache(k.data_ptr(), self.v_pages.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                                        _ptr(pos), self.page_table.data_ptr()))


def alloc_quant_cache(p: PagedParams, page_table, positions: bool = False) -> QuantCache:
    """alloc_paged_cache in 8 bits: every row stands for zeros."""
    dev = page_table.device
    pages = lambda: torch.zeros(p._pages, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.ones(p._positions, dtype=torch.uint8, device=dev)  # noqa: E731
    return QuantCache(p, pages(), pages(), scale(), scale(), page_table,
                       torch.full(p._positions, -1, dtype=torch.int32, device=dev) if positions else None)


def alloc_paged_cache(p: PagedParams, page_table, positions: bool = False) -> PagedCache:
    """A cache of `p.num_pages` pages for the sequences of `page_table`; with `positions` every row starts masked."""
    dev = page_table.device
    return PagedCache(p, torch.zeros(p._pages, dtype=p.torch_dtype, device=dev),
                      torch.zeros(p._pages, dtype=p.torch_dtype, device=dev), page_table,
                      torch.full(p._positions, -1, dtype=torch.int32, device=dev) if positions else None)


def _rows(t, dev, dtype, shape, name):
    """Rows [B, heads, n, D], or [B, heads, D] for one token, with any strides but the last -> their strides."""
    s = t.stride()
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        _refuse(t, dev, dtype, shape, name)
    if s[-1] != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    return _strides(s[0], s[1], s[2] if len(s) == 4 else 0)


def ems_paged_append(p: PagedParams, cache: PagedCache, start, k, v, positions=None, new_len=None, inv_freq=None,
                     interleaved=False, q=None, q_out=None, len_out=None):
    """Append k, v [B,Hkv,N,D] ([B,Hkv,D]: one token) from row start [B] int32 of every sequence on; keys and the
    queries q [B,Hq,N,D] are rotated by inv_freq [rot/2] f32 at their positions ([B,N] or [B,Hkv,N] int32, default
    the row).  new_len [B] int32: tokens there are of the N.  -> q_out (q's shape; pass q to rotate in place), None
    without q.  len_out [B] int32 is written start + new tokens."""
    return _append(lib().ems_paged_append, "ems_paged_append", p, _in_full(cache), start, k, v, positions, new_len, inv_freq, interleaved, q,
                   q_out, len_out)


def ems_quant_append(p: PagedParams, cache: QuantCache, start, k, v, positions=None, new_len=None, inv_freq=None,
                      interleaved=False, q=None, q_out=None, len_out=None):
    """ems_paged_append to a cache in 8 bits."""
    return _append(lib().ems_quant_append, "ems_quant_append", p, _in_8_bits(cache), start, k, v, positions, new_len, inv_freq,
                   interleaved, q, q_out, len_out)


def _in_8_bits(cache):
    if not isinstance(cache, QuantCache):
        raise ValueError("cache: a QuantCache")
    return cache


def _in_full(cache):
    if isinstance(cache, QuantCache):
        raise ValueError("cache: a PagedCache (the ems_quant calls take one in 8 bits)")
    return cache


def _append(call, name, p, cache, start, k, v, positions, new_len, inv_freq, interleaved, q, q_out, len_out):
    dev, dt, b = _current_device(), p.torch_dtype, p.batch
    cc = cache._c(p, dev)
    single = k.dim() == 3
    n = 1 if single else k.shape[2]
    tail = (p.head_dim,) if single else (n, p.head_dim)
    kv = (b, p.kv_heads) + tail
    ks, vs = _rows(k, dev, dt, kv, "k"), _rows(v, dev, dt, kv, "v")
    _check_dense(start, dev, torch.int32, (b,), "start")
    if new_len is not None:
        _check_dense(new_len, dev, torch.int32, (b,), "new_len")
    if len_out is not None:
        _check_dense(len_out, dev, torch.int32, (b,), "len_out")
    ps = None
    if positions is not None:
        shared = positions.dim() == 2
        ps_shape = (b, n) if shared else (b, p.kv_heads, n)
        if positions.shape != ps_shape or positions.dtype != torch.int32 or positions.get_device() != dev:
            _refuse(positions, dev, torch.int32, ps_shape, "positions")
        s = positions.stride()
        ps = _strides(s[0], 0 if shared else s[1], s[-1])
    rot = 0
    if inv_freq is not None:
        rot = 2 * inv_freq.shape[0]
        _check_dense(inv_freq, dev, torch.float32, (rot // 2,), "inv_freq")
    qs = qos = None
    if q is not None:
        qt = (b, p.q_heads) + tail
        qs = _rows(q, dev, dt, qt, "q")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        qos = qs if q_out is q else _rows(q_out, dev, dt, qt, "q_out")
        if not q_out.is_contiguous() and any(m > 1 and step == 0 for m, step in zip(q_out.shape, q_out.stride())):
            raise ValueError("q_out: every row in a place of its own")
    elif q_out is not None:
        raise ValueError("q_out without q")
    rc = call(C.byref(p._c), cc, n, start.data_ptr(), _ptr(new_len), k.data_ptr(), ks, v.data_ptr(), vs,
              _ptr(positions), ps, _ptr(inv_freq), rot, 1 if interleaved else 0, _ptr(q), qs,
              _ptr(q_out), qos, _ptr(len_out), _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, name)
    return q_out


def ems_paged_workspace_bytes(p: PagedParams) -> int:
    n = C.c_size_t(0)
    rc = lib().ems_paged_workspace_bytes(C.byref(p._c), C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_paged_workspace_bytes")
    return int(n.value)


def ems_paged_attention(p: PagedParams, cache: PagedCache, lens, q, want_lse=False, ws=None, out=None):
    """Attention of one new token per sequence, q [B,Hq,D], over the first lens [B] int32 rows of its pages
    -> out [B,Hq,D] (or (out, lse [B,Hq] f32) with want_lse).  `out`: (out, lse or None) to write to."""
    return _attend(lib().ems_paged_attention, "ems_paged_attention", ems_paged_workspace_bytes, p, _in_full(cache), lens, q, want_lse, ws, out)


def ems_quant_workspace_bytes(p: PagedParams) -> int:
    n = C.c_size_t(0)
    rc = lib().ems_quant_workspace_bytes(C.byref(p._c), C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_quant_workspace_bytes")
    return int(n.value)


def ems_quant_attention(p: PagedParams, cache: QuantCache, lens, q, want_lse=False, ws=None, out=None):
    """ems_paged_attention over a cache in 8 bits."""
    return _attend(lib().ems_quant_attention, "ems_quant_attention", ems_quant_workspace_bytes, p, _in_8_bits(cache), lens, q, want_lse, ws, out)


def _attend(call, name, need, p, cache, lens, q, want_lse, ws, out):
    dev = _current_device()
    cc = cache._c(p, dev)
    qs = _rows(q, dev, p.torch_dtype, p._q_row, "q")
    _check_dense(lens, dev, torch.int32, (p.batch,), "lens")
    ws = _check_ws(ws, dev, need, p)
    o, lse = _attention_out(out, dev, want_lse, p._q_row, p.torch_dtype)
    rc = call(C.byref(p._c), cc, lens.data_ptr(), q.data_ptr(), qs, o.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(), _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, name)
    return (o, lse) if want_lse else o


def ems_quant_read(p: PagedParams, cache: QuantCache, lens, rows=None, out=None):
    """The values that the first lens [B] int32 rows of every sequence stand for -> k, v [B,Hkv,rows,D], rows: all that the
    table has, or fewer; what is behind a length is left as it is (zeros in new tensors).  `out`: (k, v) to write to, of
    any strides."""
    dev = _current_device()
    cc = _in_8_bits(cache)._c(p, dev)
    _check_dense(lens, dev, torch.int32, (p.batch,), "lens")
    if out is None:
        n = p.max_pages * p.page_size if rows is None else rows
        shape = (p.batch, p.kv_heads, n, p.head_dim)
        out = tuple(torch.zeros(shape, dtype=p.torch_dtype, device="cuda") for _ in range(2))
    k, v = out
    if k.dim() != 4 or (rows is not None and k.shape[2] != rows):
        raise ValueError("out: k and v [B, Hkv, rows, D]")
    shape = (p.batch, p.kv_heads, k.shape[2], p.head_dim)
    ks, vs = (_out_rows(t, dev, p.torch_dtype, shape, name) for t, name in ((k, "k"), (v, "v")))
    rc = lib().ems_quant_read(C.byref(p._c), cc, k.shape[2], lens.data_ptr(), k.data_ptr(), ks, v.data_ptr(), vs, _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_quant_read")
    return k, v


def _out_rows(t, dev, dtype, shape, name):
    """Rows to write to: with strides like those of _rows, but no row in two places."""
    s = _rows(t, dev, dtype, shape, name)
    if not t.is_contiguous() and any(m > 1 and step == 0 for m, step in zip(t.shape, t.stride())):
        raise ValueError(f"{name}: every row in a place of its own")
    return s


def _out_like(q):
    """A new tensor of q's shape, heads and tokens in the order that q has them in."""
    d = q.dim() - 3
    swap = q.shape[d + 1] > 1 and q.shape[d] > 1 and q.stride(d + 1) > q.stride(d)
    if not swap:
        return torch.empty(q.shape, dtype=q.dtype, device=q.device)
    shape = list(q.shape)
    shape[d], shape[d + 1] = shape[d + 1], shape[d]
    return torch.empty(shape, dtype=q.dtype, device=q.device).transpose(d, d + 1)


def ems_paged_chunk_workspace_bytes(p: PagedParams, n_new: int) -> int:
    n = C.c_size_t(0)
    rc = lib().ems_paged_chunk_workspace_bytes(C.byref(p._c), n_new, C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_paged_chunk_workspace_bytes")
    return int(n.value)


def ems_paged_chunk_attention(p: PagedParams, cache: PagedCache, lens, q, new_len=None, want_lse=False, ws=None, out=None):
    """Attention of the newest tokens of every sequence, q [B,Hq,N,D] of any strides, over the first lens [B] int32 rows of
    its pages, theirs the last of them: each sees the rows up to its own.  new_len [B] int32: tokens there are of the N.
    -> out [B,Hq,N,D], heads and tokens in q's order (or (out, lse [B,Hq,N] f32) with want_lse); what is behind new_len is left
    as it is.  `out`: (out of any strides, lse or None) to write to."""
    dev = _current_device()
    cc = _in_full(cache)._c(p, dev)
    if q.dim() != 4:
        raise ValueError("q: [B, Hq, N, D]")
    n = q.shape[2]
    shape = (p.batch, p.q_heads, n, p.head_dim)
    qs = _rows(q, dev, p.torch_dtype, shape, "q")
    _check_dense(lens, dev, torch.int32, (p.batch,), "lens")
    if new_len is not None:
        _check_dense(new_len, dev, torch.int32, (p.batch,), "new_len")
    if ws is None:
        ws = torch.empty(max(ems_paged_chunk_workspace_bytes(p, n), 256), dtype=torch.uint8, device="cuda")
    else:
        _check_ws(ws, dev, None, p)
    o, lse = _many_out(out, q, dev, want_lse, shape, p.torch_dtype)
    rc = lib().ems_paged_chunk_attention(C.byref(p._c), cc, n, lens.data_ptr(), _ptr(new_len), q.data_ptr(), qs, o.data_ptr(),
                                         _out_rows(o, dev, p.torch_dtype, shape, "out"), _ptr(lse), ws.data_ptr(), ws.numel(), _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_paged_chunk_attention")
    return (o, lse) if want_lse else o


def _many_out(out, q, dev, want_lse, shape, dtype):
    if out is None:
        return _out_like(q), torch.empty(shape[:-1], dtype=torch.float32, device="cuda") if want_lse else None
    o, lse = out
    if not want_lse:
        return o, None
    if lse is None:
        raise ValueError("out: a tensor for the log-sum-exp is wanted")
    _check_dense(lse, dev, torch.float32, shape[:-1], "lse")
    return o, lse


def ems_prompt_workspace_bytes(p: PromptParams) -> int:
    n = C.c_size_t(0)
    rc = lib().ems_prompt_workspace_bytes(C.byref(p._c), C.byref(n))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_prompt_workspace_bytes")
    return int(n.value)


def ems_prompt_attention(p: PromptParams, q, k, v, q_start=None, k_start=None, want_lse=False, ws=None, out=None):
    """Causal attention of whole prompts, q [B,Hq,N,D], k, v [B,Hkv,M,D] of any strides -> out [B,Hq,N,D], heads and tokens in
    q's order (or (out, lse [B,Hq,N] f32) with want_lse).  Packed, with q_start [B + 1] int32 (first rows of the sequences):
    q, out [N,Hq,D], k, v [M,Hkv,D], lse [Hq,N]; k_start: theirs, None = q_start.  Queries are the last tokens of their
    sequence's rows.  `out`: (out of any strides, lse or None) to write to."""
    dev, dt, h, hq, d = _current_device(), p.torch_dtype, p.kv_heads, p.q_heads, p.head_dim
    if q_start is not None:
        if k_start is None:
            k_start = q_start
        _check_dense(q_start, dev, torch.int32, (p.batch + 1,), "q_start")
        _check_dense(k_start, dev, torch.int32, (p.batch + 1,), "k_start")
        shape, rows, lse_shape = (p.q_rows, hq, d), (p.k_rows, h, d), (hq, p.q_rows)
        strides, checked = _token_rows, _token_out_rows
    else:
        if k_start is not None:
            raise ValueError("k_start without q_start")
        shape, rows, lse_shape = (p.batch, hq, p.q_rows, d), (p.batch, h, p.k_rows, d), (p.batch, hq, p.q_rows)
        strides, checked = _rows, _out_rows
    qs, ks, vs = strides(q, dev, dt, shape, "q"), strides(k, dev, dt, rows, "k"), strides(v, dev, dt, rows, "v")
    if ws is None:
        ws = torch.empty(max(ems_prompt_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
    else:
        _check_ws(ws, dev, None, p)
    if out is None and q_start is not None:
        out = torch.empty(shape, dtype=dt, device="cuda"), torch.empty(lse_shape, dtype=torch.float32, device="cuda") if want_lse else None
    o, lse = _many_out(out, q, dev, want_lse, lse_shape + (d,), dt)
    rc = lib().ems_prompt_attention(C.byref(p._c), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, _ptr(q_start), _ptr(k_start),
                                    o.data_ptr(), checked(o, dev, dt, shape, "out"), _ptr(lse), ws.data_ptr(), ws.numel(), _stream_of(dev))
    if rc != EMS_OK:
        raise EmsError(rc, "ems_prompt_attention")
    return (o, lse) if want_lse else o


def _token_rows(t, dev, dtype, shape, name):
    """Rows [tokens, heads, D] with any strides but the last -> their strides."""
    s = t.stride()
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        _refuse(t, dev, dtype, shape, name)
    if s[-1] != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    return _strides(0, s[1], s[0])


def _token_out_rows(t, dev, dtype, shape, name):
    s = _token_rows(t, dev, dtype, shape, name)
    if not t.is_contiguous() and any(m > 1 and step == 0 for m, step in zip(t.shape, t.stride())):
        raise ValueError(f"{name}: every row in a place of its own")
    return s
