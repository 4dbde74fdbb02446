"""Checks of arguments that the operators' bindings share: tensors on one GPU, the stream of that GPU, addresses and strides of rows.

For single tokens the host's part of a call is longer than the kernel, so what is as it should be takes one comparison of each kind (a call of rotary positions for 64
tokens 13.1 -> 8.8 us, of norms 14.5 -> 9.1)."""
from __future__ import annotations

import torch

from . import ChunkAttnError

_only_gpu = None
BF16, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


def _refuse(name, dtype, shape, what):
    raise ValueError(f"{name}: expected a {what}{dtype} GPU tensor of shape {list(shape)}")


def rows(t, dtype, shape, inner, name):
    """Address of a GPU tensor of this type and shape whose rows are contiguous (`inner`: the strides of a row's dimensions) and the rows' stride in elements;
    (None, 0) for None."""
    if t is None:
        return None, 0
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == shape):
        _refuse(name, dtype, shape, "")
    strides = t.stride()
    if strides[1:] != inner and not all(n == 1 or s == i for n, s, i in zip(shape[1:], strides[1:], inner)):
        raise ValueError(f"{name}: the elements of a row have to be contiguous")
    if shape[0] > 1:
        return t.data_ptr(), strides[0]
    return t.data_ptr(), shape[1] * inner[0]  # (the stride of a single row says nothing)


def whole(t, dtype, shape, name):
    """Address of a contiguous GPU tensor of this type and shape; None for None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        _refuse(name, dtype, shape, "contiguous ")
    return t.data_ptr()


def given(t, dtype, shape, name):
    """The same for a tensor that has to be there."""
    try:
        if t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:  # (not a tensor)
        pass
    _refuse(name, dtype, shape, "contiguous ")


def room(workspace):
    """Address and size of a workspace; (None, 0) for None."""
    if workspace is None:
        return None, 0
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.dtype == U8 and workspace.dim() == 1 and workspace.is_contiguous()):
        _refuse("workspace", U8, ("*",), "contiguous ")
    return workspace.data_ptr(), workspace.shape[0]


def call(function, tensors, stream, *args):
    """Calls a function of the library on the GPU that holds the tensors (which need not be the current one), on `stream` or that GPU's current one."""
    global _only_gpu
    if _only_gpu is None:
        _only_gpu = torch.cuda.device_count() == 1
    if _only_gpu:  # (all of them are on it)
        rc = function(*args, torch._C._cuda_getCurrentRawStream(0) if stream is None else stream.cuda_stream)
        if rc != 0:
            raise ChunkAttnError(rc)
        return
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError("the tensors are on different GPUs")
    current = torch._C._cuda_getDevice()
    device = devices.pop() if devices else current
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(device)
    else:
        if stream.device.index != device:
            raise ValueError("the stream belongs to another GPU than the tensors")
        handle = stream.cuda_stream
    if device == current:
        rc = function(*args, handle)
    else:
        with torch.cuda.device(device):
            rc = function(*args, handle)
    if rc != 0:
        raise ChunkAttnError(rc)
