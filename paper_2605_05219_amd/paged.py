"""ctypes binding of the paged key/value cache (include/attn_paged.h): argument marshalling only.

Pools are device tensors [n_pages][H_kv][page_rows][d] (k bf16, v fp16) and [n_pages][H_kv][page_rows] (w fp32), unit
stride inside a page; the stride of the first dimension is passed on.  Index arrays and page tables are host sequences."""
from __future__ import annotations

import ctypes

import numpy as np

from .attention import attn_shape
from .binding import GDN_BF16, GDN_F32, GdnError, _check, _dp, _h32, _hp, _stream_ptr, lib

_i32, _i64, _vp, _f32, _f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_double

EXPORTS = ["attn_rope_freqs", "attn_paged_workspace_bytes", "attn_rope_append", "attn_paged_prefill", "attn_key_weights", "attn_evict"]


class attn_pages(ctypes.Structure):
    _fields_ = [("page_stride", _i64), ("n_pages", _i32), ("page_rows", _i32)]


class attn_rope(ctypes.Structure):
    _fields_ = [("rot", _i32), ("layout", _i32), ("in_dtype", _i32), ("amplitude", _f32), ("freq", _vp)]


def make_attn_rope(freqs, layout="half", amplitude=1.0, in_dtype="bf16") -> attn_rope:
    """freqs: the rot / 2 angles per position (kept alive by the result); layout "half" (pairs p, p + rot/2) or
    "interleaved" (2p, 2p + 1)."""
    f = np.ascontiguousarray(np.asarray(freqs, dtype=np.float64))
    code = {"f32": GDN_F32, "bf16": GDN_BF16, GDN_F32: GDN_F32, GDN_BF16: GDN_BF16}
    rope = attn_rope(2 * f.size, {"half": 0, "interleaved": 1}[layout], code[in_dtype], float(amplitude), f.ctypes.data if f.size else None)
    rope._freqs = f
    return rope


_ready = False


def _lib():
    global _ready
    L = lib()
    if not _ready:
        sh, pg = ctypes.POINTER(attn_shape), ctypes.POINTER(attn_pages)
        L.attn_rope_freqs.argtypes = [_i32, _f64, _i32, _f64, _f64, _f64, _f64, _vp, _vp]
        L.attn_paged_workspace_bytes.restype = _i64
        L.attn_paged_workspace_bytes.argtypes = [sh, _i32, _i64, _i64]
        L.attn_rope_append.argtypes = ([sh, ctypes.POINTER(attn_rope)] + [_vp, _i64] * 3 + [_i32] + [_vp] * 3 + [pg] + [_vp] * 4
                                       + [_vp, _vp, _i64, _vp])
        L.attn_paged_prefill.argtypes = [sh, _vp, _vp, _i32, _vp, _vp, pg] + [_vp] * 6 + [_vp, _i64, _vp]
        L.attn_key_weights.argtypes = [sh, _vp, _vp, _i32, _vp, _vp, pg] + [_vp] * 3 + [_f32, _vp, _vp, _i64] + [_vp, _i64, _vp]
        L.attn_evict.argtypes = [sh, _i32] + [_vp] * 4 + [pg] + [_vp] * 3 + [_i64] + [_vp] * 5 + [_vp, _i64, _vp]
        for f in (L.attn_rope_freqs, L.attn_rope_append, L.attn_paged_prefill, L.attn_key_weights, L.attn_evict):
            f.restype = _i32
        _ready = True
    return L


def _pages(*pools) -> attn_pages:
    """The common geometry of the given key and value pools."""
    p = pools[0]
    geo = (int(p.stride(0)), int(p.shape[0]), int(p.shape[2]))
    for x in pools[1:]:
        if (int(x.stride(0)), int(x.shape[0]), int(x.shape[2])) != geo:
            raise GdnError(-3, "pools of one geometry")
    return attn_pages(*geo)


def _table(page_cu, page_ids):
    return _h32(page_cu), _h32(page_ids)


def _ws(workspace):
    return _dp(workspace), int(workspace.numel() * workspace.element_size()) if workspace is not None else 0


KINDS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3}


def attn_rope_freqs(rot: int, base: float = 10000.0, kind: str = "plain", factor: float = 1.0, context: float = 0.0, fast: float = 32.0,
                    slow: float = 1.0):
    """See include/attn_paged.h: (the rot / 2 angles per position as float64, the amplitude).  Host only."""
    out, amp = np.zeros(max(int(rot), 0) // 2, np.float64), _f64(0.0)
    _check(_lib().attn_rope_freqs(int(rot), float(base), KINDS[kind], float(factor), float(context), float(fast), float(slow), _hp(out),
                                  ctypes.byref(amp)), "attn_rope_freqs")
    return out, amp.value


def attn_paged_workspace_bytes(shape: attn_shape, n_req: int, total_tokens: int, n_page_ids: int) -> int:
    return _check(int(_lib().attn_paged_workspace_bytes(ctypes.byref(shape), int(n_req), int(total_tokens), int(n_page_ids))),
                  "attn_paged_workspace_bytes")


def attn_rope_append(shape: attn_shape, rope: attn_rope, q, k, v, cu_seqlens, pos, start, k_pool, v_pool, page_cu, page_ids, q_out,
                     workspace, stream=None) -> None:
    """See include/attn_paged.h.  q, k, v are [T][heads][d] tensors whose token stride is passed on (heads and elements packed);
    pos may be None."""
    cu, st = _h32(cu_seqlens), _h32(start)
    ps = _h32(pos) if pos is not None else None
    tcu, ids = _table(page_cu, page_ids)
    pages = _pages(k_pool, v_pool)
    _check(_lib().attn_rope_append(ctypes.byref(shape), ctypes.byref(rope), _dp(q), int(q.stride(0)), _dp(k), int(k.stride(0)), _dp(v),
                                   int(v.stride(0)), int(st.size), _hp(cu), _hp(ps), _hp(st), ctypes.byref(pages), _dp(k_pool),
                                   _dp(v_pool), _hp(tcu), _hp(ids), _dp(q_out), *_ws(workspace), _stream_ptr(stream)), "attn_rope_append")


def attn_paged_prefill(shape: attn_shape, q, out_gate, cu_seqlens, start, k_pool, v_pool, page_cu, page_ids, o, lse, workspace,
                       stream=None) -> None:
    """See include/attn_paged.h.  out_gate and lse may be None."""
    cu, st = _h32(cu_seqlens), _h32(start)
    tcu, ids = _table(page_cu, page_ids)
    pages = _pages(k_pool, v_pool)
    _check(_lib().attn_paged_prefill(ctypes.byref(shape), _dp(q), _dp(out_gate), int(st.size), _hp(cu), _hp(st), ctypes.byref(pages),
                                     _dp(k_pool), _dp(v_pool), _hp(tcu), _hp(ids), _dp(o), _dp(lse), *_ws(workspace),
                                     _stream_ptr(stream)), "attn_paged_prefill")


def attn_key_weights(shape: attn_shape, q, lse, cu_seqlens, start, k_pool, page_cu, page_ids, decay, w_in, w_out, workspace,
                     stream=None) -> None:
    """See include/attn_paged.h.  w_in may be None or w_out; the two have one page stride."""
    cu, st = _h32(cu_seqlens), _h32(start)
    tcu, ids = _table(page_cu, page_ids)
    pages = _pages(k_pool)
    if w_in is not None and int(w_in.stride(0)) != int(w_out.stride(0)):
        raise GdnError(-3, "attn_key_weights: w_in and w_out of one geometry")
    _check(_lib().attn_key_weights(ctypes.byref(shape), _dp(q), _dp(lse), int(st.size), _hp(cu), _hp(st), ctypes.byref(pages),
                                   _dp(k_pool), _hp(tcu), _hp(ids), float(decay), _dp(w_in), _dp(w_out), int(w_out.stride(0)),
                                   *_ws(workspace), _stream_ptr(stream)), "attn_key_weights")


def attn_evict(shape: attn_shape, rows, keep, first, recent, k_pool, v_pool, w_pool, page_cu, page_ids, new_page_cu, new_page_ids, index,
               workspace, stream=None) -> None:
    """See include/attn_paged.h.  index: int32, H_kv entries per kept row."""
    rw, kp, fi, rc = _h32(rows), _h32(keep), _h32(first), _h32(recent)
    tcu, ids = _table(page_cu, page_ids)
    ncu, nids = _table(new_page_cu, new_page_ids)
    pages = _pages(k_pool, v_pool)
    _check(_lib().attn_evict(ctypes.byref(shape), int(rw.size), _hp(rw), _hp(kp), _hp(fi), _hp(rc), ctypes.byref(pages), _dp(k_pool),
                             _dp(v_pool), _dp(w_pool), int(w_pool.stride(0)), _hp(tcu), _hp(ids), _hp(ncu), _hp(nids), _dp(index),
                             *_ws(workspace), _stream_ptr(stream)), "attn_evict")
