"""ctypes binding of the residual stream's norms (include/gdn_block.h): argument marshalling only."""
from __future__ import annotations

import ctypes

from .binding import GDN_BF16, GDN_F32, _check, lib
from .rows import _dp, _here, _ld, _stream_ptr

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


_types = {}


def _dtype(code):
    if not _types:
        import torch
        _types.update({GDN_BF16: torch.bfloat16, GDN_F32: torch.float32})
    return _types.get(code)


def gdn_block_norm(shape: gdn_block_shape, y, gate, w_post, b_post, r, w_pre, b_pre, s, x, stream=None) -> None:
    """See include/gdn_block.h.  y, r, s, x (and a gate per element) are [T][D] tensors with unit inner stride, whose row stride is passed
    on; a gate per token is [T]; w, b and a gate per channel are fp32 [D].  y or r, and s or x, may be None."""
    of = y if y is not None else r
    if of is None or len(of.shape) != 2:
        raise ValueError("gdn_block_norm: y or r is needed, [T][D]")
    D, size = shape.D, of.shape
    T = size[0]
    element = shape.gate == 1
    code = shape.in_dtype
    for t, c in ((y, code), (r, shape.s_dtype), (s, shape.s_dtype), (x, shape.x_dtype), (gate if element else None, code)):
        if t is not None and (t.shape != size or size[1] != D or t.dtype is not _dtype(c)):
            raise ValueError("gdn_block_norm: tensors are [T][D], of the types that the shape says")
    for t in (w_post, b_post, w_pre, b_pre, gate if shape.gate == 3 else None):
        if t is not None and (t.numel() != D or t.dtype is not _dtype(GDN_F32) or not t.is_contiguous()):
            raise ValueError("gdn_block_norm: weights, biases and a gate per channel are fp32 [D]")
    ldg = 0
    if shape.gate == 2 and gate is not None:
        if gate.shape != size[:1] or gate.dtype is not _dtype(code):
            raise ValueError("gdn_block_norm: a gate per token is [T], of y's type")
        ldg = gate.stride(0) if T > 1 else 1
    elif element and gate is not None:
        ldg = _ld(gate)
    device = _here(y, gate, w_post, b_post, r, w_pre, b_pre, s, x)
    _check(_lib().gdn_block_norm(ctypes.byref(shape), _dp(y), _ld(y), _dp(gate), ldg, _dp(w_post), _dp(b_post), _dp(r), _ld(r), _dp(w_pre),
                                 _dp(b_pre), _dp(s), _ld(s), _dp(x), _ld(x), T, _stream_ptr(stream, device)), "gdn_block_norm")
