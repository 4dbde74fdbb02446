"""Python binding of the norms around a block with gate and residual scale (include/fused_norm.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import BF16, F32, call, room, rows, torch, whole

GATES = {"plain": 0, "sigmoid": 1, "silu": 2}
_bound = False


class Norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("gate_kind", ctypes.c_int32), ("residual_is_f32", ctypes.c_int32),
                ("weight_is_f32", ctypes.c_int32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float), ("block_scale", ctypes.c_float),
                ("y", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("y_stride", ctypes.c_int64),
                ("gate_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64), ("post_weight", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p)]


def _bind():
    global _bound
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    np = ctypes.POINTER(Norm)
    _lib.fused_norm_fwd.argtypes = [np] + [vp, i64] * 2 + [vp]
    _lib.fused_norm_fwd.restype = ctypes.c_int
    _lib.fused_norm_bwd_workspace_bytes.argtypes = [i64, i32, ctypes.POINTER(sz)]
    _lib.fused_norm_bwd_workspace_bytes.restype = ctypes.c_int
    _lib.fused_norm_bwd.argtypes = [np] + [vp, i64] * 6 + [vp, vp, i32, vp, sz, vp]
    _lib.fused_norm_bwd.restype = ctypes.c_int
    _bound = True


def _common(y, gate, first, residual_type, post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale):
    """The shared description, with the shape of `first`."""
    if not _bound:
        _bind()
    if not isinstance(first, torch.Tensor) or first.dim() != 2:
        raise ValueError("y or residual: expected a tensor [rows, cols]")
    if gate is None:
        gate_kind = "plain"  # (not looked at)
    elif gate_kind not in GATES:
        raise ValueError(f"gate_kind: expected one of {sorted(GATES)}")
    shape = first.shape
    weight = post_weight if post_weight is not None else pre_weight
    wtype = F32 if weight is None or weight.dtype == F32 else BF16
    y_at, y_stride = rows(y, BF16, shape, (1,), "y")
    gate_at, gate_stride = rows(gate, BF16, shape, (1,), "gate")
    return shape, Norm(shape[0], shape[1], GATES[gate_kind], residual_type == F32, wtype == F32, eps, residual_scale, block_scale, y_at, gate_at, None, y_stride,
                       gate_stride, 0, whole(post_weight, wtype, shape[1:], "post_weight"), whole(pre_weight, wtype, shape[1:], "pre_weight"))


def _type(*like):
    """The residual's type: that of the first tensor there is."""
    for t in like:
        if t is not None:
            return F32 if t.dtype == F32 else BF16
    return BF16


def fused_norm_fwd(y, gate, residual, post_weight, pre_weight, residual_out, h, eps=1e-6, gate_kind="sigmoid", residual_scale=1.0, block_scale=1.0,
                   stream=None) -> None:
    """residual_out = residual_scale * residual + block_scale * act(gate) * N(y; post_weight), h = N(residual_out; pre_weight).  Tensors [rows, cols] (rows may be
    strided); any of them may be None as include/fused_norm.h says.  gate_kind: "plain", "sigmoid" or "silu"."""
    rtype = _type(residual, residual_out)
    shape, d = _common(y, gate, y if y is not None else residual, rtype, post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale)
    d.residual, d.residual_stride = rows(residual, rtype, shape, (1,), "residual")
    call(_lib.fused_norm_fwd, (y, gate, residual, post_weight, pre_weight, residual_out, h), stream, ctypes.byref(d),
         *rows(residual_out, rtype, shape, (1,), "residual_out"), *rows(h, BF16, shape, (1,), "h"))


def fused_norm_bwd_workspace_bytes(num_rows, cols) -> int:
    if not _bound:
        _bind()
    n = ctypes.c_size_t(0)
    rc = _lib.fused_norm_bwd_workspace_bytes(num_rows, cols, ctypes.byref(n))
    if rc != 0:
        raise ChunkAttnError(rc)
    return n.value


def alloc_workspace(num_rows, cols, device="cuda"):
    """A uint8 tensor large enough for fused_norm_bwd at this size."""
    return torch.empty(max(fused_norm_bwd_workspace_bytes(num_rows, cols), 256), dtype=torch.uint8, device=device)


def fused_norm_bwd(y, gate, residual_out, post_weight, pre_weight, d_residual_out, d_h, dy, d_gate, d_residual, d_post_weight, d_pre_weight, workspace,
                   eps=1e-6, gate_kind="sigmoid", residual_scale=1.0, block_scale=1.0, accumulate_weights=False, stream=None) -> None:
    """Gradients of fused_norm_fwd from those of its outputs; residual_out is what the forward wrote.  Gradients of weights are float32 [cols], written
    or added to; outputs that are None are not formed.  workspace may be None without gradients of weights."""
    rtype = _type(residual_out, d_residual_out, d_residual)
    first = y if y is not None else residual_out if residual_out is not None else d_residual_out
    shape, d = _common(y, gate, first, rtype, post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale)
    one = (1,)
    call(_lib.fused_norm_bwd,
         (y, gate, residual_out, post_weight, pre_weight, d_residual_out, d_h, dy, d_gate, d_residual, d_post_weight, d_pre_weight, workspace), stream,
         ctypes.byref(d), *rows(residual_out, rtype, shape, one, "residual_out"), *rows(d_residual_out, rtype, shape, one, "d_residual_out"),
         *rows(d_h, BF16, shape, one, "d_h"), *rows(dy, BF16, shape, one, "dy"), *rows(d_gate, BF16, shape, one, "d_gate"),
         *rows(d_residual, rtype, shape, one, "d_residual"), whole(d_post_weight, F32, shape[1:], "d_post_weight"), whole(d_pre_weight, F32, shape[1:], "d_pre_weight"),
         bool(accumulate_weights), *room(workspace))
