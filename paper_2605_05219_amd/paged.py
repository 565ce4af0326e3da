"""ctypes binding of the paged key/value cache (include/attn_paged.h): argument marshalling only.

Pools are device tensors [n_pages][H_kv][page_rows][d] (k bf16, v fp16) and [n_pages][H_kv][page_rows] (w fp32), packed
inside a page; the stride of the first dimension is passed on.  Index arrays and page tables are host sequences."""
from __future__ import annotations

import ctypes

import numpy as np

from .attention import attn_shape
from .binding import GDN_BF16, GDN_F32, GdnError, _check, _hp, lib
from .binding import _stream_ptr as _stream_object_ptr

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


def _stream_ptr(stream=None):
    """The given stream's handle, or the current one's without an object made for it (3 us a call)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(torch.cuda.current_device()) if stream is None and raw is not None else _stream_object_ptr(stream)


def _dp(x):
    """A device tensor's (or None's) address: a plain number, of which the call's argument types make a pointer (a tenth of a microsecond less)."""
    return x.data_ptr() if x is not None else None


_ints = ctypes.c_int32 * 0
_from_buffer = _ints.from_buffer
_INT32 = np.dtype(np.int32)


def _ip(a):
    """An int32 array as an argument that the call reads in place (a fifth of what `_hp` takes)."""
    try:
        return _from_buffer(a)
    except (TypeError, ValueError, BufferError):          # read-only, or with gaps
        return _from_buffer(np.array(a, order="C"))


def _array(n, x):
    """A host sequence of n entries as an argument."""
    a = np.asarray(x, _INT32)
    if a.size != n:
        raise ValueError("index arrays have inconsistent lengths")
    return _ip(a)


def _tokens(n, cu):
    """The new tokens of n requests, and their offsets as an argument."""
    a = np.asarray(cu, _INT32)
    if a.size != n + 1:
        raise ValueError("index arrays have inconsistent lengths")
    return a.item(n), _ip(a)


def _table(n, cu, ids):
    """The offsets of n requests, and the page ids that they say, as arguments."""
    a, b = np.asarray(cu, _INT32), np.asarray(ids, _INT32)
    if a.size != n + 1 or b.size < a.item(n):
        raise ValueError("index arrays have inconsistent lengths")
    return _ip(a), _ip(b)


def _holds(count, *tensors):
    """Refuses tensors (or None) of fewer elements than the call reads or writes."""
    for x in tensors:
        if x is not None and x.numel() < count:
            raise GdnError(-3, f"{count} elements are needed, not {x.numel()}")


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


_types = {}                                              # "bf16", "f16", "f32", "i32", and the codes of the first and the third


def _typed(want, *tensors):
    """Refuses tensors (or None) of another type than the kernels read."""
    if not _types:
        import torch
        _types.update({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32, GDN_BF16: torch.bfloat16, GDN_F32: torch.float32})
    want = _types.get(want)                              # (None: a code that the call itself refuses)
    for x in tensors:
        if getattr(x, "dtype", want) is not want and want is not None:
            raise GdnError(-3, f"a tensor of {want} is needed, not of {x.dtype}")


def _packed(*tensors):
    for x in tensors:
        if x is not None and not x.is_contiguous():
            raise GdnError(-3, "a tensor without gaps and in order is needed")


def _ld(x):
    """The token stride of [T][heads][d] (or [T][heads * d]) whose tokens are packed; that of a single token is nobody's."""
    stride, size = x.stride(), x.shape
    if stride[-1] != 1 or (len(size) == 3 and stride[1] != size[2] and size[1] > 1):
        raise GdnError(-3, "a token's heads and elements are packed")
    return stride[0] if size[0] > 1 else size[-1] * (size[1] if len(size) == 3 else 1)


def _inside(stride, size):
    """Whether a pool's pages are packed inside."""
    rest = 1
    for i in range(len(size) - 1, 0, -1):
        if stride[i] != rest and size[i] > 1:
            return False
        rest *= size[i]
    return True


def _pages(shape, *pools):
    """The common geometry of the given key and value pools."""
    p = pools[0]
    stride, size = p.stride(), p.shape
    for x in pools[1:]:
        if x.stride() != stride or x.shape != size:
            raise GdnError(-3, "pools of one geometry")
    n, heads, rows, d = size
    if ((stride[3] != 1 or stride[2] != d or stride[1] != rows * d) and not _inside(stride, size)) or heads != shape.H_kv or d != shape.d:
        raise GdnError(-3, "a page is packed: [H_kv][page_rows][d]")
    return ctypes.byref(attn_pages(stride[0], n, rows))


def _weights_stride(w, k_pool):
    stride = w.stride()
    if w.shape != k_pool.shape[:3] or not _inside(stride, w.shape):
        raise GdnError(-3, "a page of weights is packed, and there is one for every page of keys: [H_kv][page_rows]")
    return stride[0]


def _ws(workspace):
    return _dp(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0


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
    _typed("bf16", k_pool, q_out)
    _typed("f16", v_pool)
    _typed(rope.in_dtype, q, k, v)
    _packed(q_out)
    n = len(start)
    tokens, cu = _tokens(n, cu_seqlens)
    _holds(tokens * shape.d * shape.H_q, q, q_out)
    _holds(tokens * shape.d * shape.H_kv, k, v)
    _check(_lib().attn_rope_append(ctypes.byref(shape), ctypes.byref(rope), _dp(q), _ld(q), _dp(k), _ld(k), _dp(v), _ld(v), n, cu,
                                   None if pos is None else _array(n, pos), _array(n, start), _pages(shape, k_pool, v_pool), _dp(k_pool), _dp(v_pool),
                                   *_table(n, page_cu, page_ids), _dp(q_out), *_ws(workspace), _stream_ptr(stream)), "attn_rope_append")


def attn_paged_prefill(shape: attn_shape, q, out_gate, cu_seqlens, start, k_pool, v_pool, page_cu, page_ids, o, lse, workspace,
                       stream=None) -> None:
    """See include/attn_paged.h.  out_gate and lse may be None."""
    _typed("bf16", q, out_gate, k_pool)
    _typed("f16", v_pool)
    _typed("f32", lse)
    _packed(q, out_gate, o, lse)
    n, space = len(start), _ws(workspace)
    tokens, cu = _tokens(n, cu_seqlens)
    table = _table(n, page_cu, page_ids)
    _holds(tokens * shape.H_q * shape.d, q, out_gate, o)
    _holds(tokens * shape.H_q, lse)
    try:
        _typed(shape.o_dtype, o)
    except GdnError:                                     # (a workspace that is too small is what the call refuses first)
        if space[1] >= attn_paged_workspace_bytes(shape, n, max(0, tokens), max(0, int(page_cu[-1]))):
            raise
    _check(_lib().attn_paged_prefill(ctypes.byref(shape), _dp(q), _dp(out_gate), n, cu, _array(n, start), _pages(shape, k_pool, v_pool), _dp(k_pool), _dp(v_pool),
                                     *table, _dp(o), _dp(lse), *space, _stream_ptr(stream)), "attn_paged_prefill")


def attn_key_weights(shape: attn_shape, q, lse, cu_seqlens, start, k_pool, page_cu, page_ids, decay, w_in, w_out, workspace,
                     stream=None) -> None:
    """See include/attn_paged.h.  w_in may be None or w_out; the two have one page stride."""
    _typed("bf16", q, k_pool)
    _typed("f32", lse, w_in, w_out)
    _packed(q, lse)
    w_stride = _weights_stride(w_out, k_pool)
    if w_in is not None and w_in is not w_out and _weights_stride(w_in, k_pool) != w_stride:
        raise GdnError(-3, "attn_key_weights: w_in and w_out of one geometry")
    n = len(start)
    tokens, cu = _tokens(n, cu_seqlens)
    _holds(tokens * shape.H_q * shape.d, q)
    _holds(tokens * shape.H_q, lse)
    _check(_lib().attn_key_weights(ctypes.byref(shape), _dp(q), _dp(lse), n, cu, _array(n, start), _pages(shape, k_pool), _dp(k_pool),
                                   *_table(n, page_cu, page_ids), float(decay), _dp(w_in), _dp(w_out), w_stride, *_ws(workspace), _stream_ptr(stream)),
           "attn_key_weights")


def attn_evict(shape: attn_shape, rows, keep, first, recent, k_pool, v_pool, w_pool, page_cu, page_ids, new_page_cu, new_page_ids, index,
               workspace, stream=None) -> None:
    """See include/attn_paged.h.  index: int32, H_kv entries per kept row."""
    _typed("bf16", k_pool)
    _typed("f16", v_pool)
    _typed("f32", w_pool)
    _typed("i32", index)
    _packed(index)
    n, rows, keep = len(rows), np.asarray(rows, _INT32), np.asarray(keep, _INT32)
    if rows.size == keep.size:
        _holds(int(np.minimum(rows, keep).sum(dtype=np.int64)) * shape.H_kv, index)
    _check(_lib().attn_evict(ctypes.byref(shape), n, _array(n, rows), _array(n, keep), _array(n, first), _array(n, recent), _pages(shape, k_pool, v_pool),
                             _dp(k_pool), _dp(v_pool), _dp(w_pool), _weights_stride(w_pool, k_pool), *_table(n, page_cu, page_ids),
                             *_table(n, new_page_cu, new_page_ids), _dp(index), *_ws(workspace), _stream_ptr(stream)), "attn_evict")
