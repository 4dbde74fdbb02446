"""Python binding of attention over a paged cache (include/paged_attn.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import BF16, F32, I32, call, given, room, rows, torch, whole
from .paged_cache import CACHE_TYPES

_bound = False


class Desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_q_heads", "num_kv_heads", "head_dim", "num_seqs", "total_q", "page_size", "num_pages", "max_pages", "cache_type")] + [
        ("softmax_scale", ctypes.c_float)]


def _bind():
    global _bound
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    _lib.paged_attn_validate.argtypes = [dp]
    _lib.paged_attn_validate.restype = ctypes.c_int
    _lib.paged_attn_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    _lib.paged_attn_workspace_bytes.restype = ctypes.c_int
    _lib.paged_attn_fwd.argtypes = [dp, vp, i64] + [vp] * 7 + [vp, i64, vp, vp, sz, vp]
    _lib.paged_attn_fwd.restype = ctypes.c_int
    _bound = True


def make_desc(num_q_heads, num_kv_heads, head_dim, num_seqs, total_q, page_size, num_pages, max_pages, softmax_scale, cache_type="bf16"):
    """Builds a paged_attn_desc; cache_type "bf16" or "e4m3"."""
    if not _bound:
        _bind()
    if cache_type not in CACHE_TYPES:
        raise ValueError(f"cache_type: one of {sorted(CACHE_TYPES)}")
    d = Desc(num_q_heads, num_kv_heads, head_dim, num_seqs, total_q, page_size, num_pages, max_pages, CACHE_TYPES[cache_type][0], float(softmax_scale))
    d._dtype = CACHE_TYPES[cache_type][1]
    return d


def paged_attn_validate(desc) -> int:
    return _lib.paged_attn_validate(ctypes.byref(desc))


def paged_attn_workspace_bytes(desc) -> int:
    n = ctypes.c_size_t(0)
    rc = _lib.paged_attn_workspace_bytes(ctypes.byref(desc), ctypes.byref(n))
    if rc != 0:
        raise ChunkAttnError(rc)
    return n.value


def alloc_workspace(desc, device="cuda"):
    """A uint8 tensor large enough for paged_attn_fwd on this descriptor."""
    return torch.empty(max(paged_attn_workspace_bytes(desc), 256), dtype=torch.uint8, device=device)


def paged_attn_fwd(desc, q, k_cache, v_cache, table, kv_len, q_start, o, lse, workspace, k_scale=None, v_scale=None, stream=None) -> None:
    """Attention of q [total_q, num_q_heads, head_dim] over the pages of each sequence (table [num_seqs, max_pages], kv_len [num_seqs], q_start [num_seqs + 1], all int32);
    writes o like q and, unless it is None, lse [num_q_heads, total_q] float32.  k_scale, v_scale [num_kv_heads] float32 for cache_type "e4m3"."""
    H, Hk, d, n = desc.num_q_heads, desc.num_kv_heads, desc.head_dim, desc.num_seqs
    dtype = desc._dtype
    scale = whole if dtype == BF16 else given
    qs, cs = (desc.total_q, H, d), (desc.num_pages, Hk, desc.page_size, d)
    call(_lib.paged_attn_fwd, (q, k_cache, v_cache, k_scale, v_scale, table, kv_len, q_start, o, lse, workspace), stream, ctypes.byref(desc), *rows(q, BF16, qs, (d, 1), "q"),
         given(k_cache, dtype, cs, "k_cache"), given(v_cache, dtype, cs, "v_cache"), scale(k_scale, F32, (Hk,), "k_scale"), scale(v_scale, F32, (Hk,), "v_scale"),
         given(table, I32, (n, desc.max_pages), "table"), given(kv_len, I32, (n,), "kv_len"), given(q_start, I32, (n + 1,), "q_start"), *rows(o, BF16, qs, (d, 1), "o"),
         whole(lse, F32, (H, desc.total_q), "lse"), *room(workspace))
