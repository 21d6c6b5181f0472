"""What the torch forms of the library's calls have in common: checks of
tensors, the stream a call runs on, workspace sizes."""

from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding as B

_TYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}

# A call on few rows lasts as long as its marshalling: the current stream's
# handle is asked for directly (torch.cuda.current_stream takes 2 us) and sizes are
# kept.  Every output has a storage of its own (1.4 us each; a view of a common one 0.9), so
# that a loss that is kept keeps no workspace.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _address(t):
    return None if t is None else t.data_ptr()


def _vector(name, t, dtype, shape, device):
    """Refuses what is not a contiguous tensor of that type and shape on that device."""
    try:
        if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
            return
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _matrix(name, t, of="classes"):
    """(rows, columns, pitch) of a tensor whose rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or t.dtype not in _TYPES:
        raise ValueError(f"{name} must be [rows, {of}] in float32 or bfloat16")
    rows, classes = t.shape
    pitch, step = t.stride()
    if classes < 1:
        raise ValueError(f"{name} must have {of}")
    if classes > 1 and step != 1:
        raise ValueError(f"rows of {name} must be contiguous")
    if rows < 2:
        return rows, classes, classes
    if pitch < classes:
        raise ValueError(f"rows of {name} overlap")
    return rows, classes, pitch


def _on(device, stream, tensors, call):
    """call(stream handle) with the device and stream current; tensors given
    are kept from reuse until a stream that is not current is past the call."""
    if stream is None and device.index == torch.cuda.current_device():
        return call(_raw_stream(device.index))
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else \
            torch.cuda.default_stream(device)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors are on {device}")
    with torch.cuda.stream(stream):
        result = call(stream.cuda_stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return result


@functools.lru_cache(maxsize=4096)
def _bytes(query, *sizes):
    n = C.c_int64()
    B._check(getattr(B.lib, query)(*sizes, C.byref(n)), query)
    return n.value
