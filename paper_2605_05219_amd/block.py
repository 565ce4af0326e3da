"""ctypes binding of the residual stream's norms (include/gdn_block.h): argument marshalling only."""
from __future__ import annotations

import ctypes

from .binding import GDN_BF16, GDN_F32, _check, lib
from .rows import _device, _packed, _rows, _stream

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float

EXPORTS = ["gdn_block_norm"]

_NORMS = {"none": 0, "rms": 1, "layer": 2}
_GATES = {"none": 0, "element": 1, "token": 2, "channel": 3}


class gdn_block_shape(ctypes.Structure):
    _fields_ = [("D", _i32), ("post", _i32), ("pre", _i32), ("in_dtype", _i32), ("s_dtype", _i32), ("x_dtype", _i32), ("gate", _i32),
                ("gate_act", _i32), ("eps_post", _f32), ("eps_pre", _f32), ("scale", _f32), ("offset", _f32)]


def make_block_shape(D, post="none", pre="rms", in_dtype="bf16", s_dtype="bf16", x_dtype="bf16", gate="none", gate_act="none", eps_post=1e-6,
                     eps_pre=1e-6, scale=1.0, offset=0.0) -> gdn_block_shape:
    """post, pre: "none", "rms" or "layer"; gate: "none", "element", "token" or "channel", itself or its "sigmoid"."""
    code = {"f32": GDN_F32, "bf16": GDN_BF16, GDN_F32: GDN_F32, GDN_BF16: GDN_BF16}
    return gdn_block_shape(int(D), _NORMS[post], _NORMS[pre], code[in_dtype], code[s_dtype], code[x_dtype], _GATES[gate],
                           {"none": 0, "sigmoid": 1}[gate_act], float(eps_post), float(eps_pre), float(scale), float(offset))


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        L.gdn_block_norm.restype = _i32
        L.gdn_block_norm.argtypes = [ctypes.POINTER(gdn_block_shape), _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i64, _vp, _i64,
                                     _i64, _vp]
        _ready = True
    return L


def gdn_block_norm_raw(shape, y=0, ldy=0, gate=0, ldg=0, w_post=0, b_post=0, r=0, ldr=0, w_pre=0, b_pre=0, s=0, lds=0, x=0, ldx=0, T=0,
                       stream_ptr=0) -> int:
    """The C entry point with plain integers for the pointers; returns the status code (no exception)."""
    return int(_lib().gdn_block_norm(ctypes.byref(shape) if shape is not None else None, y, ldy, gate, ldg, w_post, b_post, r, ldr, w_pre, b_pre,
                                     s, lds, x, ldx, T, stream_ptr))


_types = ()                                              # torch's fp32 and bf16, in the order of their codes: assigned at once, since threads' first calls may meet


def gdn_block_norm(shape: gdn_block_shape, y, gate, w_post, b_post, r, w_pre, b_pre, s, x, stream=None) -> None:
    """See include/gdn_block.h.  y, r, s, x (and a gate per element) are [T][D] tensors with unit inner stride, whose row stride is passed
    on; a gate per token is [T]; w, b and a gate per channel are fp32 [D].  y or r, and s or x, may be None."""
    global _types
    if not _types:
        import torch
        _types = (torch.float32, torch.bfloat16)
    of = y if y is not None else r
    size = of.shape if of is not None else ()
    D = shape.D
    if len(size) != 2 or size[1] != D or not (0 <= shape.in_dtype <= 1 and 0 <= shape.s_dtype <= 1 and 0 <= shape.x_dtype <= 1):
        raise ValueError("gdn_block_norm: y or r is needed, [T][D], and types that there are")
    name, f32, device, T, vector = "gdn_block_norm", _types[0], _device(), size[0], size[1:]
    wide, held = _types[shape.in_dtype], _types[shape.s_dtype]
    kind = shape.gate
    if kind == 1:
        at_gate, ldg = _rows(gate, size, wide, device, name)
    elif kind == 3:
        at_gate, ldg = _packed(gate, vector, f32, device, name), 0
    elif kind == 2 and gate is not None:
        if gate.shape != size[:1] or gate.dtype is not wide or gate.get_device() != device:
            raise ValueError("gdn_block_norm: a gate per token is [T], of y's type and on its device")
        at_gate, ldg = gate.data_ptr(), gate.stride(0) if T > 1 else 1
    else:
        at_gate, ldg = None, 0
    at_y, ldy = _rows(y, size, wide, device, name)
    at_r, ldr = _rows(r, size, held, device, name)
    at_s, lds = _rows(s, size, held, device, name)
    at_x, ldx = _rows(x, size, _types[shape.x_dtype], device, name)
    _check(_lib().gdn_block_norm(ctypes.byref(shape), at_y, ldy, at_gate, ldg, _packed(w_post, vector, f32, device, name),
                                 _packed(b_post, vector, f32, device, name), at_r, ldr, _packed(w_pre, vector, f32, device, name),
                                 _packed(b_pre, vector, f32, device, name), at_s, lds, at_x, ldx, T, _stream(stream, device)), name)
