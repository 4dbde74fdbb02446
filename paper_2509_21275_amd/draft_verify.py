"""Python binding of the verification of drafted tokens (include/draft_verify.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import BF16, F32, I32, call, given, room, torch, whole

_bound = False


def _bind():
    global _bound
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    _lib.draft_verify_workspace_bytes.argtypes = [i32] * 3 + [ctypes.POINTER(sz)]
    _lib.draft_verify_workspace_bytes.restype = ctypes.c_int
    _lib.draft_verify.argtypes = [i32] * 4 + [vp, i64, vp, i64] + [vp] * 8 + [sz, vp]
    _lib.draft_verify.restype = ctypes.c_int
    _bound = True


def draft_verify_workspace_bytes(batch, max_drafts, vocab) -> int:
    if not _bound:
        _bind()
    n = ctypes.c_size_t(0)
    rc = _lib.draft_verify_workspace_bytes(batch, max_drafts, vocab, ctypes.byref(n))
    if rc != 0:
        raise ChunkAttnError(rc)
    return n.value


def alloc_workspace(batch, max_drafts, vocab, device="cuda"):
    """A uint8 tensor large enough for draft_verify."""
    return torch.empty(max(draft_verify_workspace_bytes(batch, max_drafts, vocab), 256), dtype=torch.uint8, device=device)


def _probabilities(t, shape, dtype, name):
    """Address and stride of rows that may be apart by more than the vocabulary, by the same everywhere."""
    if t is None:
        return None, 0
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == shape):
        raise ValueError(f"{name}: expected a {dtype} GPU tensor of shape {list(shape)}")
    n, m, v = shape
    s = t.stride()
    if not (v == 1 or s[2] == 1):
        raise ValueError(f"{name}: the elements of a row have to be contiguous")
    row = s[1] if m > 1 else s[0] if n > 1 else v
    if n > 1 and m > 1 and s[0] != m * row:
        raise ValueError(f"{name}: all rows have to be equally far apart")
    return t.data_ptr(), row


def draft_verify(target, draft, tokens, count, uniforms, last_uniform, accepted, rejected, out, workspace, stream=None) -> None:
    """target [batch, max_drafts + 1, vocab] and draft [batch, max_drafts, vocab] (or None) float32 or bf16 probabilities, tokens [batch, max_drafts] int32, count [batch] int32 (or None),
    uniforms [batch, max_drafts] and last_uniform [batch] float32; writes accepted, rejected (unless it is None) [batch] and out [batch, max_drafts + 1], int32."""
    if not _bound:
        _bind()
    if not (isinstance(target, torch.Tensor) and target.dim() == 3 and target.shape[1] >= 1 and target.dtype in (F32, BF16)):
        raise ValueError("target: expected a float32 or bf16 tensor of 3 dimensions")
    n, places, V = target.shape
    K = places - 1
    call(_lib.draft_verify, (target, draft, tokens, count, uniforms, last_uniform, accepted, rejected, out, workspace), stream, n, K, V, 1 if target.dtype == F32 else 0,
         *_probabilities(target, (n, places, V), target.dtype, "target"), *_probabilities(draft, (n, K, V), target.dtype, "draft"), given(tokens, I32, (n, K), "tokens"),
         whole(count, I32, (n,), "count"), given(uniforms, F32, (n, K), "uniforms"), given(last_uniform, F32, (n,), "last_uniform"), given(accepted, I32, (n,), "accepted"),
         whole(rejected, I32, (n,), "rejected"), given(out, I32, (n, K + 1), "out"), *room(workspace))
