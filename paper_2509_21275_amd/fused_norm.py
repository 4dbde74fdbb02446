"""Python binding of the norms around a block with gate and residual scale (include/fused_norm.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes

from . import ChunkAttnError, _lib
from ._args import call, rows, whole

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


def _common(y, gate, residual_like, post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale):
    """The shared description, its shape and the residual's type.  `residual_like`: the tensors that share the residual's type."""
    import torch
    if not _bound:
        _bind()
    if gate_kind == "none" and gate is None:
        gate_kind = "plain"
    if gate_kind not in GATES:
        raise ValueError(f"gate_kind: expected one of {sorted(GATES)}")
    first = next((t for t in (y, *residual_like) if isinstance(t, torch.Tensor) and t.dim() == 2), None)
    if first is None:
        raise ValueError("y or residual: expected a tensor [rows, cols]")
    shape = tuple(first.shape)
    rtype = next((t.dtype for t in residual_like if t is not None), torch.bfloat16)
    weights = [w for w in (post_weight, pre_weight) if w is not None]
    wtype = weights[0].dtype if weights else torch.float32
    f32 = (torch.float32,)
    if rtype not in (torch.bfloat16, torch.float32) or wtype not in (torch.bfloat16, torch.float32):
        raise ValueError("residuals and weights: expected bfloat16 or float32")
    d = Norm(rows=shape[0], cols=shape[1], gate_kind=GATES[gate_kind], residual_is_f32=rtype == torch.float32, weight_is_f32=wtype == torch.float32,
             eps=eps, residual_scale=residual_scale, block_scale=block_scale)
    d.y, d.y_stride = rows(y, (torch.bfloat16,), shape, "y")
    d.gate, d.gate_stride = rows(gate, (torch.bfloat16,), shape, "gate")
    d.post_weight = whole(post_weight, (wtype,), shape[1:], "post_weight")
    d.pre_weight = whole(pre_weight, (wtype,), shape[1:], "pre_weight")
    return d, shape, (rtype,), f32


def fused_norm_fwd(y, gate, residual, post_weight, pre_weight, residual_out, h, eps=1e-6, gate_kind="sigmoid", residual_scale=1.0, block_scale=1.0,
                   stream=None) -> None:
    """residual_out = residual_scale * residual + block_scale * act(gate) * N(y; post_weight), h = N(residual_out; pre_weight).  Tensors [rows, cols] (rows may be
    strided); any of them may be None as include/fused_norm.h says.  gate_kind: "plain", "sigmoid" or "silu"."""
    import torch
    d, shape, rtype, _ = _common(y, gate, (residual, residual_out), post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale)
    d.residual, d.residual_stride = rows(residual, rtype, shape, "residual")
    call(_lib.fused_norm_fwd, (y, gate, residual, post_weight, pre_weight, residual_out, h), stream, ctypes.byref(d),
         *rows(residual_out, rtype, shape, "residual_out"), *rows(h, (torch.bfloat16,), shape, "h"))


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
    import torch
    return torch.empty(max(fused_norm_bwd_workspace_bytes(num_rows, cols), 256), dtype=torch.uint8, device=device)


def fused_norm_bwd(y, gate, residual_out, post_weight, pre_weight, d_residual_out, d_h, dy, d_gate, d_residual, d_post_weight, d_pre_weight, workspace,
                   eps=1e-6, gate_kind="sigmoid", residual_scale=1.0, block_scale=1.0, accumulate_weights=False, stream=None) -> None:
    """Gradients of fused_norm_fwd from those of its outputs; residual_out is what the forward wrote.  Gradients of weights are float32 [cols], written
    or added to; outputs that are None are not formed.  workspace may be None without gradients of weights."""
    import torch
    d, shape, rtype, f32 = _common(y, gate, (residual_out, d_residual_out, d_residual), post_weight, pre_weight, eps, gate_kind, residual_scale, block_scale)
    bf16 = (torch.bfloat16,)
    if workspace is not None:
        whole(workspace, (torch.uint8,), (None,), "workspace")
    call(_lib.fused_norm_bwd,
         (y, gate, residual_out, post_weight, pre_weight, d_residual_out, d_h, dy, d_gate, d_residual, d_post_weight, d_pre_weight, workspace), stream,
         ctypes.byref(d), *rows(residual_out, rtype, shape, "residual_out"), *rows(d_residual_out, rtype, shape, "d_residual_out"), *rows(d_h, bf16, shape, "d_h"),
         *rows(dy, bf16, shape, "dy"), *rows(d_gate, bf16, shape, "d_gate"), *rows(d_residual, rtype, shape, "d_residual"),
         whole(d_post_weight, f32, shape[1:], "d_post_weight"), whole(d_pre_weight, f32, shape[1:], "d_pre_weight"), int(bool(accumulate_weights)),
         None if workspace is None else workspace.data_ptr(), 0 if workspace is None else workspace.nbytes)
