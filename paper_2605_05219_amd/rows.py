"""What the bindings of row-wise operators share: row strides, addresses, the device and its stream."""
from __future__ import annotations

from .binding import _stream_ptr as _stream_object_ptr

_current = None


def _current_device():
    """The current device's number, -1 where there is none."""
    global _current
    if _current is None:
        import torch
        if not torch.cuda.is_available():
            return -1
        torch.cuda.init()
        _current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _current()


def _here(*tensors):
    """The current device, on which all tensors have to lie: a launch goes there, whatever device an address is of."""
    device = _current_device()
    for x in tensors:
        if x is not None and x.get_device() != device:
            raise ValueError(f"a tensor of the current device ({device}) is needed, not of {x.device}")
    return device


def _stream_ptr(stream, device):
    """The given stream's handle, or the current one's without an object made for it; without a device none (the launch says so)."""
    if stream is None:
        if device < 0:
            return None
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(device)
    return _stream_object_ptr(stream)


def _dp(x):
    """A device tensor's (or None's) address."""
    return x.data_ptr() if x is not None else None


def _ld(x):
    """The row stride of an [n][width] tensor whose rows are packed; that of a single row is nobody's."""
    if x is None:
        return 0
    size, stride = x.shape, x.stride()
    if stride[1] != 1 and size[1] > 1:
        raise ValueError("rows are packed: the inner stride is 1")
    return stride[0] if size[0] > 1 else -(-size[1] // 8) * 8
