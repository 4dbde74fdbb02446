"""Checks of arguments that the operators' bindings share: tensors on one GPU, the stream of that GPU, addresses and strides of rows."""
from __future__ import annotations

import contextlib

from . import ChunkAttnError


def on_gpu(t, dtypes, shape, name):
    """A GPU tensor of one of these types and of this shape (None: any size), at any strides."""
    import torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.dim() == len(shape) and all(w is None or w == n for w, n in zip(shape, t.shape))):
        kinds = " or ".join(str(d) for d in dtypes)
        raise ValueError(f"{name}: expected a {kinds} GPU tensor of shape [{', '.join('*' if w is None else str(w) for w in shape)}]")
    return t


def rows(t, dtypes, shape, name):
    """Address of a tensor whose rows [shape[1:]] are contiguous, and their stride in elements; (None, 0) for None."""
    if t is None:
        return None, 0
    on_gpu(t, dtypes, shape, name)
    inner = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != inner:
            raise ValueError(f"{name}: the elements of a row have to be contiguous")
        inner *= size
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else inner)


def whole(t, dtypes, shape, name):
    """Address of a contiguous tensor; None for None."""
    if t is None:
        return None
    if not on_gpu(t, dtypes, shape, name).is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


def call(function, tensors, stream, *args):
    """Calls a function of the library on the GPU that holds the tensors (which need not be the current one), on `stream` or that GPU's current one."""
    import torch
    device = None
    for t in tensors:
        if t is not None:
            if device is None:
                device = t.get_device()
            elif t.get_device() != device:
                raise ValueError("the tensors are on different GPUs")
    if device is None:
        device = torch._C._cuda_getDevice()
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(device)
    else:
        if stream.device.index != device:
            raise ValueError("the stream belongs to another GPU than the tensors")
        handle = stream.cuda_stream
    with contextlib.nullcontext() if device == torch._C._cuda_getDevice() else torch.cuda.device(device):
        rc = function(*args, handle)
    if rc != 0:
        raise ChunkAttnError(rc)
