"""Python binding of the paged cache's tables and of writing into it (include/paged_cache.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import BF16, F32, I32, call, given, room, rows, torch, whole

_bound = False
E4M3, I64 = torch.float8_e4m3fn, torch.int64
CACHE_TYPES = {"bf16": (0, BF16), "e4m3": (1, E4M3)}


class Desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


def _bind():
    global _bound
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    _lib.paged_cache_validate.argtypes = [dp]
    _lib.paged_cache_validate.restype = ctypes.c_int
    _lib.paged_cache_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    _lib.paged_cache_workspace_bytes.restype = ctypes.c_int
    _lib.paged_cache_extend.argtypes = [dp] + [vp] * 11 + [i32, vp, vp, sz, vp]
    _lib.paged_cache_extend.restype = ctypes.c_int
    _lib.paged_cache_truncate.argtypes = [dp] + [vp] * 10 + [sz, vp]
    _lib.paged_cache_truncate.restype = ctypes.c_int
    _lib.paged_cache_write.argtypes = [i32] * 6 + [vp, i64, vp, i64] + [vp] * 6
    _lib.paged_cache_write.restype = ctypes.c_int
    _bound = True


def make_desc(num_requests, max_pages, page_size, num_pages):
    """Builds a paged_cache_desc."""
    if not _bound:
        _bind()
    return Desc(num_requests, max_pages, page_size, num_pages)


def paged_cache_validate(desc) -> int:
    return _lib.paged_cache_validate(ctypes.byref(desc))


def paged_cache_workspace_bytes(desc) -> int:
    n = ctypes.c_size_t(0)
    rc = _lib.paged_cache_workspace_bytes(ctypes.byref(desc), ctypes.byref(n))
    if rc != 0:
        raise ChunkAttnError(rc)
    return n.value


def alloc_workspace(desc, device="cuda"):
    """A uint8 tensor large enough for paged_cache_extend and paged_cache_truncate on this descriptor."""
    return torch.empty(max(paged_cache_workspace_bytes(desc), 256), dtype=torch.uint8, device=device)


def paged_cache_extend(desc, new_tokens, kv_len, held, table, free_pages, num_free, kv_len_out, held_out, num_free_out, q_start, slots, granted, workspace,
                       stream=None) -> None:
    """Pages and slots for new_tokens [num_requests] tokens of each request; writes the state behind the call (kv_len_out, held_out, num_free_out, which may be the inputs, and new
    entries of table), q_start [num_requests + 1], slots [rows] int64 (its length is the most rows there are) and, unless it is None, granted [num_requests]."""
    n, one = (desc.num_requests,), (1,)
    if not (isinstance(slots, torch.Tensor) and slots.dim() == 1):
        raise ValueError("slots: expected a tensor of one dimension")
    call(_lib.paged_cache_extend, (new_tokens, kv_len, held, table, free_pages, num_free, kv_len_out, held_out, num_free_out, q_start, slots, granted, workspace), stream,
         ctypes.byref(desc), given(new_tokens, I32, n, "new_tokens"), given(kv_len, I32, n, "kv_len"), given(held, I32, n, "held"),
         given(table, I32, (desc.num_requests, desc.max_pages), "table"), given(free_pages, I32, (desc.num_pages,), "free_pages"), given(num_free, I32, one, "num_free"),
         given(kv_len_out, I32, n, "kv_len_out"), given(held_out, I32, n, "held_out"), given(num_free_out, I32, one, "num_free_out"),
         given(q_start, I32, (desc.num_requests + 1,), "q_start"), given(slots, I64, slots.shape, "slots"), slots.shape[0], whole(granted, I32, n, "granted"), *room(workspace))


def paged_cache_truncate(desc, drop, kv_len, held, table, free_pages, num_free, kv_len_out, held_out, num_free_out, workspace, stream=None) -> None:
    """Takes drop [num_requests] tokens off the end of each request and puts pages that hold none of those left back on the stack; *_out may be the inputs."""
    n, one = (desc.num_requests,), (1,)
    call(_lib.paged_cache_truncate, (drop, kv_len, held, table, free_pages, num_free, kv_len_out, held_out, num_free_out, workspace), stream, ctypes.byref(desc),
         given(drop, I32, n, "drop"), given(kv_len, I32, n, "kv_len"), given(held, I32, n, "held"), given(table, I32, (desc.num_requests, desc.max_pages), "table"),
         given(free_pages, I32, (desc.num_pages,), "free_pages"), given(num_free, I32, one, "num_free"), given(kv_len_out, I32, n, "kv_len_out"),
         given(held_out, I32, n, "held_out"), given(num_free_out, I32, one, "num_free_out"), *room(workspace))


def paged_cache_write(k, v, slots, k_cache, v_cache, k_scale=None, v_scale=None, stream=None) -> None:
    """Keys and values k, v [rows, num_kv_heads, head_dim] bf16 (rows may be apart, as in a projection's output) to slots [rows] int64 of k_cache, v_cache [num_pages, num_kv_heads,
    page_size, head_dim], bf16 or float8_e4m3fn; k_scale, v_scale [num_kv_heads] float32 (float8_e4m3fn only)."""
    if not _bound:
        _bind()
    if not (isinstance(k, torch.Tensor) and k.dim() == 3 and isinstance(v, torch.Tensor) and isinstance(k_cache, torch.Tensor) and k_cache.dim() == 4
            and isinstance(slots, torch.Tensor) and isinstance(v_cache, torch.Tensor)):
        raise ValueError("k, v, slots, k_cache, v_cache: expected tensors, k of 3 and k_cache of 4 dimensions")
    n, H, d = k.shape
    pages, page = k_cache.shape[0], k_cache.shape[2]
    dtype = E4M3 if k_cache.dtype == E4M3 else BF16
    scale = given if dtype == E4M3 else whole
    cs, ks = (pages, H, page, d), (n, H, d)
    call(_lib.paged_cache_write, (k, v, slots, k_cache, v_cache, k_scale, v_scale), stream, n, H, d, page, pages, 1 if dtype == E4M3 else 0, *rows(k, BF16, ks, (d, 1), "k"),
         *rows(v, BF16, ks, (d, 1), "v"), given(slots, I64, (n,), "slots"), scale(k_scale, F32, (H,), "k_scale"), scale(v_scale, F32, (H,), "v_scale"),
         given(k_cache, dtype, cs, "k_cache"), given(v_cache, dtype, cs, "v_cache"))
