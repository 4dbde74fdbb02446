"""Python binding of the rotary positions of a chunk (include/chunk_rope.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, Desc, _lib
from ._args import BF16, F32, call, rows

SCALINGS = {"none": 0, "linear": 1, "base": 2, "ramp": 3}
_bound = False


class Rope(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("frequencies", ctypes.POINTER(ctypes.c_double)),
                ("magnitude", ctypes.c_float)]


def _bind():
    global _bound
    vp, i64, i32, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
    dp, rp = ctypes.POINTER(Desc), ctypes.POINTER(Rope)
    _lib.chunk_rope_frequencies.argtypes = [i32, dbl, i32, dbl, dbl, dbl, dbl, ctypes.POINTER(dbl)]
    _lib.chunk_rope_frequencies.restype = ctypes.c_int
    _lib.chunk_rope_fwd.argtypes = [dp, rp] + [vp, i64] * 4 + [vp]
    _lib.chunk_rope_fwd.restype = ctypes.c_int
    _lib.chunk_rope_bwd.argtypes = [dp, rp, vp, i64, vp, i64, i32, vp, i64, vp, i64, vp]
    _lib.chunk_rope_bwd.restype = ctypes.c_int
    _bound = True


def rope_frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0, original_length=0, low_rotations=1.0, high_rotations=32.0):
    """The angles per position (radians) of the rotary_dim / 2 pairs, as a list; see CHUNK_ROPE_* for the scalings."""
    if not _bound:
        _bind()
    if scaling not in SCALINGS:
        raise ValueError(f"scaling: expected one of {sorted(SCALINGS)}")
    out = (ctypes.c_double * max(1, int(rotary_dim) // 2))()
    rc = _lib.chunk_rope_frequencies(int(rotary_dim), float(base), SCALINGS[scaling], float(factor), float(original_length), float(low_rotations),
                                     float(high_rotations), out)
    if rc != 0:
        raise ChunkAttnError(rc)
    return list(out)


def make_rope(rotary_dim, base=10000.0, interleaved=False, scaling="none", factor=1.0, original_length=0, low_rotations=1.0, high_rotations=32.0,
              magnitude=1.0, frequencies=None):
    """Builds a chunk_rope_desc, with the frequencies of rope_frequencies or the caller's own; keep it for as long as calls use it."""
    if frequencies is None:
        frequencies = rope_frequencies(rotary_dim, base, scaling, factor, original_length, low_rotations, high_rotations)
    if len(frequencies) != int(rotary_dim) // 2:
        raise ValueError("frequencies: expected rotary_dim / 2 values")
    arr = (ctypes.c_double * max(1, len(frequencies)))(*[float(f) for f in frequencies])
    r = Rope(int(rotary_dim), 1 if interleaved else 0, arr, float(magnitude))
    r._keepalive = arr
    return r


def chunk_rope_fwd(desc, rope, q, k, q_out, k_out, stream=None) -> None:
    """q [total_q, num_q_heads, head_dim], k [total_q, num_kv_heads, head_dim] (rows may be strided) to q_out, of q's shape, and to the chunk's own rows
    of k_out [total_kv, num_kv_heads, head_dim].  Either pair may be None."""
    if not _bound:
        _bind()
    d, n, heads, inner = desc.head_dim, desc.total_q, desc.num_kv_heads, (desc.head_dim, 1)
    qs = (n, desc.num_q_heads, d)
    call(_lib.chunk_rope_fwd, (q, k, q_out, k_out), stream, ctypes.byref(desc), ctypes.byref(rope), *rows(q, BF16, qs, inner, "q"),
         *rows(k, BF16, (n, heads, d), inner, "k"), *rows(q_out, BF16, qs, inner, "q_out"), *rows(k_out, BF16, (desc.total_kv, heads, d), inner, "k_out"))


def chunk_rope_bwd(desc, rope, dq, dk, dq_out, dk_out, stream=None) -> None:
    """Gradients back: dq to dq_out, the chunk's own rows of dk [total_kv, num_kv_heads, head_dim] (bf16 or float32) to dk_out [total_q, num_kv_heads,
    head_dim], both bf16.  Either pair may be None."""
    if not _bound:
        _bind()
    d, n, heads, inner = desc.head_dim, desc.total_q, desc.num_kv_heads, (desc.head_dim, 1)
    qs, f32 = (n, desc.num_q_heads, d), dk is not None and dk.dtype == F32
    call(_lib.chunk_rope_bwd, (dq, dk, dq_out, dk_out), stream, ctypes.byref(desc), ctypes.byref(rope), *rows(dq, BF16, qs, inner, "dq"),
         *rows(dk, F32 if f32 else BF16, (desc.total_kv, heads, d), inner, "dk"), f32, *rows(dq_out, BF16, qs, inner, "dq_out"),
         *rows(dk_out, BF16, (n, heads, d), inner, "dk_out"))
