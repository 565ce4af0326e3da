"""What the bindings of row-wise operators share: a tensor's checks with what the call needs of it, the device and its stream.

A call of one token takes the GPU two or three microseconds, so each of these is a single pass over a tensor's properties."""
from __future__ import annotations

from .binding import _stream_ptr as _stream_object_ptr

_current = _raw_stream = None


def _device():
    """The current device's number, on which a launch goes; -1 where there is none."""
    global _current, _raw_stream
    if _current is None:
        import torch
        if not torch.cuda.is_available():
            return -1
        torch.cuda.init()
        _current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return _current()


def _stream(stream, device):
    """The given stream's handle, or the current one's without an object made for it; without a device none (the launch says so)."""
    if stream is None:
        if device < 0:
            return None
        if _raw_stream is not None:
            return _raw_stream(device)
    if getattr(stream, "device_index", device) != device:
        raise ValueError(f"a stream of device {device} is needed, not of {stream.device}")
    return _stream_object_ptr(stream)


def _rows(x, size, dtype, device, what):
    """(address, row stride) of an [n][width] tensor of the given size, type and device, whose rows are packed; (None, 0) of None.  The stride of a
    single row is nobody's: the width's next multiple of 8 stands for it."""
    if x is None:
        return None, 0
    stride = x.stride()
    if x.shape != size or x.dtype is not dtype or x.get_device() != device or (stride[1] != 1 and size[1] > 1):
        raise ValueError(f"{what}: a tensor of {dtype} {tuple(size)} with packed rows on device {device} is needed, not of {x.dtype} {tuple(x.shape)} "
                         f"with strides {tuple(stride)} on {x.device}")
    return x.data_ptr(), stride[0] if size[0] > 1 else -(-size[1] // 8) * 8


def _packed(x, size, dtype, device, what):
    """The address of a tensor of the given size, type and device without gaps; None of None."""
    if x is None:
        return None
    if x.shape != size or x.dtype is not dtype or x.get_device() != device or not x.is_contiguous():
        raise ValueError(f"{what}: a tensor of {dtype} {tuple(size)} without gaps on device {device} is needed, not of {x.dtype} {tuple(x.shape)} "
                         f"with strides {tuple(x.stride())} on {x.device}")
    return x.data_ptr()
