"""ctypes binding of the mixture of experts (include/gdn_moe.h): argument marshalling only."""
from __future__ import annotations

import ctypes

from .binding import GDN_BF16, GDN_F32, _check, lib
from .linear import ACTS
from .rows import _device, _packed, _rows, _stream

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float

EXPORTS = ["gdn_moe_workspace_bytes", "gdn_moe", "gdn_moe_tune"]

_SCORES = {"softmax": 0, "sigmoid": 1}


class gdn_moe_shape(ctypes.Structure):
    _fields_ = [("E", _i32), ("k", _i32), ("D", _i32), ("F", _i32), ("act", _i32), ("score", _i32), ("normalise", _i32), ("router_dtype", _i32),
                ("routed_scale", _f32)]


def make_moe_shape(E, k, D, F, act="silu", score="softmax", normalise=True, routed_scale=1.0, router_dtype="bf16") -> gdn_moe_shape:
    """E experts of which a token takes k; D channels, F of an expert; act: one of linear.ACTS; score: "softmax" or "sigmoid"."""
    code = {"f32": GDN_F32, "bf16": GDN_BF16, GDN_F32: GDN_F32, GDN_BF16: GDN_BF16}
    return gdn_moe_shape(int(E), int(k), int(D), int(F), ACTS[act], _SCORES[score], int(bool(normalise)), code[router_dtype], float(routed_scale))


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        sh = ctypes.POINTER(gdn_moe_shape)
        L.gdn_moe_workspace_bytes.restype = _i64
        L.gdn_moe_workspace_bytes.argtypes = [sh, _i64]
        L.gdn_moe.restype = _i32
        L.gdn_moe.argtypes = [sh, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp]
        L.gdn_moe_tune.restype = _i32
        L.gdn_moe_tune.argtypes = [_i32]
        _ready = True
    return L


def gdn_moe_workspace_bytes(shape: gdn_moe_shape, T: int) -> int:
    return _check(int(_lib().gdn_moe_workspace_bytes(ctypes.byref(shape), int(T))), "gdn_moe_workspace_bytes")


def gdn_moe_raw(shape, x=0, ldx=0, w_router=0, choice_bias=0, w_gate_up=0, w_down=0, add=0, ld_add=0, y=0, ldy=0, ids=0, weights=0, T=0, workspace=0,
                workspace_bytes=0, stream_ptr=0) -> int:
    """The C entry point with plain integers for the pointers; returns the status code (no exception)."""
    return int(_lib().gdn_moe(ctypes.byref(shape) if shape is not None else None, x, ldx, w_router, choice_bias, w_gate_up, w_down, add, ld_add, y, ldy,
                              ids, weights, T, workspace, workspace_bytes, stream_ptr))


_types = ()                                              # torch's fp32, bf16 and int32: assigned at once, since threads' first calls may meet


def gdn_moe(shape: gdn_moe_shape, x, w_router, choice_bias, w_gate_up, w_down, add, y, ids, weights, workspace, stream=None) -> None:
    """See include/gdn_moe.h.  x, add, y: bf16 [T][D] with unit inner stride, whose row stride is passed on; w_router [E][D] (bf16 or fp32, as the shape
    says), w_gate_up [E][2 F][D] and w_down [E][D][F] bf16, choice_bias fp32 [E], ids int32 and weights fp32 [T][k], all without gaps.
    choice_bias, add, ids and weights may be None."""
    global _types
    if not _types:
        import torch
        _types = (torch.float32, torch.bfloat16, torch.int32)
    f32, bf16, i32 = _types
    name, size, device = "gdn_moe", x.shape, _device()
    E, k, D, F = shape.E, shape.k, shape.D, shape.F
    if len(size) != 2 or size[1] != D:
        raise ValueError("gdn_moe: x is [T][D]")
    T = size[0]
    at_x, ldx = _rows(x, size, bf16, device, name)
    at_add, ld_add = _rows(add, size, bf16, device, name)
    at_y, ldy = _rows(y, size, bf16, device, name)
    room = 0
    if workspace is not None:
        room = workspace.numel() * workspace.element_size()
        if not workspace.is_contiguous() or workspace.get_device() != device:
            raise ValueError("gdn_moe: a workspace without gaps on the tensors' device")
    _check(_lib().gdn_moe(ctypes.byref(shape), at_x, ldx, _packed(w_router, (E, D), f32 if shape.router_dtype == GDN_F32 else bf16, device, name),
                          _packed(choice_bias, (E,), f32, device, name), _packed(w_gate_up, (E, 2 * F, D), bf16, device, name),
                          _packed(w_down, (E, D, F), bf16, device, name), at_add, ld_add, at_y, ldy, _packed(ids, (T, k), i32, device, name),
                          _packed(weights, (T, k), f32, device, name), T, workspace.data_ptr() if room else None, room, _stream(stream, device)), name)


def gdn_moe_tune(shape: int) -> int:
    """Fixes the kernels of the experts' products (see include/gdn_moe.h) or returns the choice to the library (-1); returns the previous setting."""
    return int(_lib().gdn_moe_tune(int(shape)))
