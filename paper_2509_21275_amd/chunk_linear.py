"""Python binding of linear attention with a decay for each head (include/chunk_linear.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import BF16, F32, I32, call, room, torch, whole

_bound = False


class Seg(ctypes.Structure):
    _fields_ = [("start", ctypes.c_int32), ("len", ctypes.c_int32), ("state_in", ctypes.c_int32), ("state_out", ctypes.c_int32)]


class Desc(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("total", ctypes.c_int32),
                ("num_states", ctypes.c_int32), ("num_segments", ctypes.c_int32), ("segments", ctypes.POINTER(Seg)), ("scale", ctypes.c_float)]


def _bind():
    global _bound
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    _lib.chunk_linear_validate.argtypes = [dp]
    _lib.chunk_linear_validate.restype = ctypes.c_int
    _lib.chunk_linear_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    _lib.chunk_linear_workspace_bytes.restype = ctypes.c_int
    _lib.chunk_linear_fwd.argtypes = [dp] + [vp] * 8 + [sz, vp]
    _lib.chunk_linear_fwd.restype = ctypes.c_int
    _lib.chunk_linear_bwd.argtypes = [dp] + [vp] * 12 + [sz, vp]
    _lib.chunk_linear_bwd.restype = ctypes.c_int
    _lib.chunk_linear_step.argtypes = [i32] * 4 + [vp] * 6 + [i32, vp, vp, ctypes.c_float, vp]
    _lib.chunk_linear_step.restype = ctypes.c_int
    _bound = True


def make_desc(segs, num_q_heads, num_kv_heads, head_dim, total, num_states, scale):
    """Builds a chunk_linear_desc of segments (start, len, state_in, state_out), slots -1 where there is no state; keep the returned object alive for the
    duration of the call."""
    if not _bound:
        _bind()
    arr = (Seg * max(1, len(segs)))(*[Seg(*[int(x) for x in s]) for s in segs])
    d = Desc(num_q_heads, num_kv_heads, head_dim, total, num_states, len(segs), arr, float(scale))
    d._keepalive = arr
    return d


def chunk_linear_validate(desc) -> int:
    return _lib.chunk_linear_validate(ctypes.byref(desc))


def chunk_linear_workspace_bytes(desc):
    f, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    rc = _lib.chunk_linear_workspace_bytes(ctypes.byref(desc), ctypes.byref(f), ctypes.byref(b))
    if rc != 0:
        raise ChunkAttnError(rc)
    return f.value, b.value


def alloc_workspace(desc, device="cuda"):
    """A uint8 tensor large enough for both chunk_linear_fwd and chunk_linear_bwd on this descriptor."""
    return torch.empty(max(*chunk_linear_workspace_bytes(desc), 256), dtype=torch.uint8, device=device)


def _shapes(desc):
    d, Hk = desc.head_dim, desc.num_kv_heads
    return (desc.total, desc.num_q_heads, d), (desc.total, Hk, d), (Hk,), (desc.num_states, Hk, d, d)


def chunk_linear_fwd(desc, q, k, v, log_decay, states_in, o, states_out, workspace, stream=None) -> None:
    """Writes o [total, num_q_heads, head_dim] and the states that segments leave in states_out [num_states, num_kv_heads, head_dim, head_dim]; states_in and
    states_out may be None where no segment names a slot, or the same tensor."""
    qs, ks, hs, ss = _shapes(desc)
    call(_lib.chunk_linear_fwd, (q, k, v, log_decay, states_in, o, states_out, workspace), stream, ctypes.byref(desc), whole(q, BF16, qs, "q"), whole(k, BF16, ks, "k"),
         whole(v, BF16, ks, "v"), whole(log_decay, F32, hs, "log_decay"), whole(states_in, F32, ss, "states_in"), whole(o, BF16, qs, "o"),
         whole(states_out, F32, ss, "states_out"), *room(workspace))


def chunk_linear_bwd(desc, q, k, v, log_decay, states_in, d_o, d_states_out, dq, dk, dv, d_states_in, workspace, stream=None) -> None:
    """Writes dq, dk, dv and, if it is given, d_states_in; d_states_out (gradients of the states left, None: zeros)."""
    qs, ks, hs, ss = _shapes(desc)
    call(_lib.chunk_linear_bwd, (q, k, v, log_decay, states_in, d_o, d_states_out, dq, dk, dv, d_states_in, workspace), stream, ctypes.byref(desc), whole(q, BF16, qs, "q"),
         whole(k, BF16, ks, "k"), whole(v, BF16, ks, "v"), whole(log_decay, F32, hs, "log_decay"), whole(states_in, F32, ss, "states_in"), whole(d_o, BF16, qs, "d_o"),
         whole(d_states_out, F32, ss, "d_states_out"), whole(dq, BF16, qs, "dq"), whole(dk, BF16, ks, "dk"), whole(dv, BF16, ks, "dv"),
         whole(d_states_in, F32, ss, "d_states_in"), *room(workspace))


def chunk_linear_step(q, k, v, log_decay, states_in, states_out, slots, o, scale, stream=None) -> None:
    """One token for each of a batch: q, o [batch, num_q_heads, head_dim], k, v [batch, num_kv_heads, head_dim], slots int32 [batch] into states_in and states_out
    [num_states, num_kv_heads, head_dim, head_dim], which may be the same tensor."""
    if not _bound:
        _bind()
    if not (isinstance(q, torch.Tensor) and q.dim() == 3 and isinstance(k, torch.Tensor) and k.dim() == 3 and isinstance(states_in, torch.Tensor) and states_in.dim() == 4):
        raise ValueError("q, k, states_in: expected tensors of 3, 3 and 4 dimensions")
    B, H, d = q.shape
    Hk, n = k.shape[1], states_in.shape[0]
    ks, ss = (B, Hk, d), (n, Hk, d, d)
    call(_lib.chunk_linear_step, (q, k, v, log_decay, states_in, states_out, slots, o), stream, B, H, Hk, d, whole(q, BF16, (B, H, d), "q"), whole(k, BF16, ks, "k"),
         whole(v, BF16, ks, "v"), whole(log_decay, F32, (Hk,), "log_decay"), whole(states_in, F32, ss, "states_in"), whole(states_out, F32, ss, "states_out"), n,
         whole(slots, I32, (B,), "slots"), whole(o, BF16, (B, H, d), "o"), float(scale))
