"""The paged key/value cache (include/attn_paged.h) against its oracle.

CPU part: exports, the frequencies, the refusals.  GPU part (marked gpu), through the C ABI, on pools whose unused rows and
pages hold NaN.  The tolerances, from the roundings (half a step: bf16 2^-8, fp16 2^-11, fp32 2^-24 relative):

  rotated q, k  2^-8 |ref| for the store, and 2^-20 amplitude (|x| + |y|) for the angle (2^-25 of a turn from its fp32 value),
                cosine, sine and three fp32 roundings; values are numpy's own float16 conversion, bit for bit
  o             every weight is off by 2^-11 at most and they are normalised by their own sum: 2 * 2^-11 max |v - o| <= 2^-9 max |v|,
                twice the step for what the fp32 sums add (2^-8 max |v|), and 2^-8 |ref| for a bf16 store
  lse           a logit is a sum of d products in fp32, (d + 16) 2^-24 scale sum |q_i k_i|, and so is their log-sum-exp; 2^-20 (1 + |lse|) for
                the exponentials, the logarithm and the scaling
  weights       each term off by e^x - 1 with x the error of a logit and of lse in fp32 (2^-22 |lse|), and rows 2^-24 for the sum
  eviction      copies: bit for bit
"""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import attn_oracle as ao, paged_oracle as po
from paper_2605_05219_amd import attention as AT, binding as B, paged as PG, workloads as wl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ----------------------------------------------------------------------------- host
def test_library_exports_every_symbol_the_paged_header_declares():
    header = open(os.path.join(ROOT, "include", "attn_paged.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(attn_\w+)\s*\(", header))
    assert declared == set(PG.EXPORTS)
    L = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert getattr(L, name) is not None


@pytest.mark.parametrize("rot", [2, 16, 64, 128, 256])
@pytest.mark.parametrize("kw", [dict(), dict(kind="linear", factor=8.0), dict(kind="base", factor=4.0), dict(kind="ramp", factor=16.0, context=4096.0),
                                dict(kind="ramp", factor=2.0, context=100.0, fast=8.0, slow=0.5), dict(kind="ramp", factor=1.0, context=10.0)])
def test_frequencies_are_the_formulas(rot, kw):
    if rot == 2 and kw.get("kind") == "base":
        with pytest.raises(B.GdnError):
            PG.attn_rope_freqs(rot, **kw)
        return
    f, a = PG.attn_rope_freqs(rot, 10000.0, **kw)
    rf, ra = po.rope_freqs(rot, 10000.0, **kw)
    np.testing.assert_allclose(f, rf, rtol=1e-13)
    assert a == pytest.approx(ra, rel=1e-15)
    assert PG.attn_rope_freqs(0)[0].size == 0


@pytest.mark.parametrize("args,kw", [((15,), {}), ((-2,), {}), ((16, 1.0), {}), ((16, float("nan")), {}), ((16, 1e4), dict(kind="linear", factor=0.5)),
                                     ((16, 1e4), dict(kind="ramp", factor=2.0, context=0.0)), ((16, 1e4), dict(kind="base", factor=float("inf"))),
                                     ((16, 1e4), dict(kind="ramp", factor=2.0, context=100.0, fast=1.0, slow=1.0))])
def test_frequencies_refuse(args, kw):
    with pytest.raises(B.GdnError) as ei:
        PG.attn_rope_freqs(*args, **kw)
    assert ei.value.code == -3


class FakePool:
    """Stands in for a device tensor: the checks under test return before any pointer is used."""

    def __init__(self, ptr=0x10000, shape=(40, 2, 16, 64), stride0=None, nbytes=1 << 30):
        self._ptr, self.shape, self._n = ptr, shape, nbytes
        self._s0 = int(np.prod(shape[1:])) if stride0 is None else stride0

    def data_ptr(self): return self._ptr
    def is_contiguous(self): return True

    def stride(self, i=None):
        inside = [int(np.prod(self.shape[j + 1:])) for j in range(1, len(self.shape))]
        return (self._s0, *inside) if i is None else (self._s0, *inside)[i]
    def numel(self): return self._n
    def element_size(self): return 1


K_POOL, V_POOL, W_POOL = FakePool(0x200000), FakePool(0x300000), FakePool(0x400000, (40, 2, 16))
X = FakePool(0x10000, (9, 4, 64))
WS = FakePool(0x100000)
CALL = dict(shape=AT.make_attn_shape(4, 2, 64), cu_seqlens=[0, 5, 9], start=[0, 20], k_pool=K_POOL, v_pool=V_POOL, page_cu=[0, 1, 3],
            page_ids=[7, 3, 39], workspace=WS)
FRONT = [                                                                     # what every call refuses
    (dict(shape=AT.make_attn_shape(4, 2, 96)), -3),
    (dict(shape=AT.make_attn_shape(4, 3, 64)), -3),
    (dict(k_pool=FakePool(0x200000, (40, 2, 24, 64)), v_pool=FakePool(0x300000, (40, 2, 24, 64))), -3),   # rows per page
    (dict(k_pool=FakePool(0x200000, (40, 2, 8, 64)), v_pool=FakePool(0x300000, (40, 2, 8, 64))), -3),
    (dict(k_pool=FakePool(0x200000, (40, 2, 512, 64)), v_pool=FakePool(0x300000, (40, 2, 512, 64))), -3),
    (dict(k_pool=FakePool(0x200000, stride0=2044), v_pool=FakePool(0x300000, stride0=2044)), -2),
    (dict(k_pool=FakePool(0x200000, stride0=1024), v_pool=FakePool(0x300000, stride0=1024)), -3),         # pages would overlap
    (dict(page_ids=[7, 3, 40]), -5),
    (dict(page_ids=[-1, 3, 39]), -5),
    (dict(k_pool=FakePool(0)), -1),
    (dict(k_pool=FakePool(0x200008)), -2),
    (dict(workspace=None), -9),
    (dict(workspace=FakePool(0x100000, nbytes=64)), -9),
    (dict(workspace=FakePool(0x100004)), -9),
]
TOKENS = FRONT + [
    (dict(cu_seqlens=[1, 5, 9]), -4),
    (dict(cu_seqlens=[0, 5, 4]), -4),
    (dict(page_cu=[1, 1, 3]), -4),
    (dict(page_cu=[0, 3, 1]), -4),
    (dict(start=[-1, 20]), -10),
    (dict(start=[0, 29]), -10),                                               # 33 rows, two pages
    (dict(start=[0, 2 ** 31 - 5]), -10),
    (dict(page_cu=[0, 0, 3]), -10),
]


def refused(fn, code, *args):
    with pytest.raises(B.GdnError) as ei:
        fn(*args)
    assert ei.value.code == code


@pytest.fixture
def no_stream(monkeypatch):
    monkeypatch.setattr(PG, "_stream_ptr", lambda s=None: ctypes.c_void_p(0))


@pytest.mark.parametrize("over,code", TOKENS + [
    (dict(page_ids=[7, 3, 3]), -6), (dict(page_ids=[39, 3, 39]), -6),         # a page that gets rows, listed twice
    (dict(page_ids=[3, 3, 39]), -6),                                          # ... among the rows another request holds
    (dict(pos=[0, -1]), -10), (dict(pos=[0, 2 ** 31 - 3]), -10),
    (dict(rope=PG.make_attn_rope(np.ones(36))), -3), (dict(rope=PG.make_attn_rope(np.ones(4))), -3),
    (dict(rope=PG.make_attn_rope(np.full(8, np.inf))), -3), (dict(rope=PG.make_attn_rope(np.ones(8), amplitude=float("nan"))), -3),
    (dict(q=FakePool(0, (9, 4, 64))), -1), (dict(k=FakePool(0x10002, (9, 2, 64))), -2), (dict(q_out=FakePool(0x10008, (9, 4, 64))), -2),
    (dict(v=FakePool(0x10000, (9, 2, 64), 132)), -2), (dict(q=FakePool(0x10000, (9, 4, 64), 128)), -3),
])
def test_rope_append_refuses(no_stream, over, code):
    a = dict(CALL, rope=PG.make_attn_rope(np.ones(32)), q=X, k=FakePool(0x10000, (9, 2, 64)), v=FakePool(0x10000, (9, 2, 64)), pos=[0, 100], q_out=X)
    a.update(over)
    refused(PG.attn_rope_append, code, a["shape"], a["rope"], a["q"], a["k"], a["v"], a["cu_seqlens"], a["pos"], a["start"], a["k_pool"], a["v_pool"],
            a["page_cu"], a["page_ids"], a["q_out"], a["workspace"])


@pytest.mark.parametrize("over,code", TOKENS + [
    (dict(q=FakePool(0, (9, 4, 64))), -1), (dict(o=FakePool(0)), -1), (dict(o=FakePool(0x10004)), -2), (dict(gate=FakePool(0x10002)), -2),
    (dict(lse=FakePool(0x10002)), -2), (dict(shape=AT.make_attn_shape(4, 2, 64, scale=0.0)), -3),
])
def test_paged_prefill_refuses(no_stream, over, code):
    a = dict(CALL, q=X, gate=None, o=X, lse=None)
    a.update(over)
    refused(PG.attn_paged_prefill, code, a["shape"], a["q"], a["gate"], a["cu_seqlens"], a["start"], a["k_pool"], a["v_pool"], a["page_cu"],
            a["page_ids"], a["o"], a["lse"], a["workspace"])


@pytest.mark.parametrize("over,code", TOKENS + [
    (dict(page_ids=[7, 7, 39]), -6), (dict(q=FakePool(0, (9, 4, 64))), -1), (dict(lse=FakePool(0)), -1), (dict(w_out=FakePool(0, (40, 2, 16))), -1),
    (dict(w_out=FakePool(0x400002, (40, 2, 16))), -2), (dict(w_in=FakePool(0x400001, (40, 2, 16))), -2), (dict(decay=float("nan")), -3),
    (dict(w_in=None, w_out=FakePool(0x400000, (40, 2, 16), 31)), -3), (dict(w_in=FakePool(0x400000, (40, 2, 16), 64)), -3),
])
def test_key_weights_refuses(no_stream, over, code):
    a = dict(CALL, q=X, lse=FakePool(0x10000), decay=1.0, w_in=W_POOL, w_out=W_POOL)
    a.update(over)
    refused(PG.attn_key_weights, code, a["shape"], a["q"], a["lse"], a["cu_seqlens"], a["start"], a["k_pool"], a["page_cu"], a["page_ids"], a["decay"],
            a["w_in"], a["w_out"], a["workspace"])


@pytest.mark.parametrize("over,code", FRONT + [
    (dict(rows=[17, 24]), -10), (dict(rows=[-1, 24]), -10), (dict(keep=[5, -1]), -10), (dict(first=[3, 2]), -10), (dict(recent=[2, 30]), -10),
    (dict(keep=[5, 17]), -10), (dict(page_cu=[0, 3, 1]), -4), (dict(new_page_cu=[1, 1, 2]), -4),
    (dict(new_page_ids=[1, 1]), -6), (dict(new_page_ids=[1, 40]), -5), (dict(new_page_ids=[1, 39]), -7), (dict(index=FakePool(0)), -1),
    (dict(index=FakePool(0x10001)), -2), (dict(v_pool=FakePool(0)), -1), (dict(w_pool=FakePool(0x400000, (40, 2, 16), 31)), -3),
])
def test_evict_refuses(no_stream, over, code):
    a = dict(CALL, rows=[5, 24], keep=[4, 10], first=[2, 2], recent=[2, 3], w_pool=W_POOL, new_page_cu=[0, 1, 2], new_page_ids=[1, 2], index=FakePool())
    a.update(over)
    refused(PG.attn_evict, code, a["shape"], a["rows"], a["keep"], a["first"], a["recent"], a["k_pool"], a["v_pool"], a["w_pool"], a["page_cu"],
            a["page_ids"], a["new_page_cu"], a["new_page_ids"], a["index"], a["workspace"])


def test_calls_with_nothing_to_do_touch_nothing(no_stream):
    sh, rope = AT.make_attn_shape(4, 2, 64), PG.make_attn_rope(np.ones(32))
    z = FakePool(0, (0, 4, 64))
    for cu, st, tcu, ids in [([0], [], [0], []), ([0, 0, 0], [0, 3], [0, 0, 1], [7])]:
        PG.attn_rope_append(sh, rope, z, z, z, cu, None, st, K_POOL, V_POOL, tcu, ids, z, None)
        PG.attn_paged_prefill(sh, z, None, cu, st, K_POOL, V_POOL, tcu, ids, z, None, None)
    PG.attn_key_weights(sh, z, z, [0, 0], [0], K_POOL, [0, 0], [], 1.0, None, W_POOL, None)
    PG.attn_evict(sh, [0, 5], [3, 0], [0, 0], [0, 0], K_POOL, V_POOL, W_POOL, [0, 0, 1], [7], [0, 0, 0], [], z, None)
    with pytest.raises(B.GdnError):
        PG.attn_paged_workspace_bytes(sh, -1, 0, 0)
    assert PG.attn_paged_workspace_bytes(sh, 3, 100, 500) > PG.attn_paged_workspace_bytes(sh, 3, 100, 0) > 0


def test_tensors_that_the_call_would_read_wrongly_are_refused(no_stream):
    """Orders and gaps that no argument of the C call says."""
    import torch
    sh, rope = AT.make_attn_shape(4, 2, 64), PG.make_attn_rope(np.ones(32))
    k, v = torch.zeros(40, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(40, 2, 16, 64, dtype=torch.float16)
    w, ws = torch.zeros(40, 2, 16), torch.zeros(1 << 10, dtype=torch.uint8)
    q, kv, lse = torch.zeros(9, 4, 64, dtype=torch.bfloat16), torch.zeros(9, 2, 64, dtype=torch.bfloat16), torch.zeros(9, 4)
    cu, st, tcu, ids = [0, 5, 9], [0, 20], [0, 1, 3], [7, 3, 39]
    turned = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    wide = lambda x: torch.zeros(*x.shape[:-1], 2 * x.shape[-1], dtype=x.dtype)[..., :x.shape[-1]]  # noqa: E731
    append = lambda q=q, k_=kv, v_=kv, kp=k, vp=v, out=q: PG.attn_rope_append(sh, rope, q, k_, v_, cu, None, st, kp, vp, tcu, ids, out, ws)  # noqa: E731
    attend = lambda q=q, gate=None, kp=k, vp=v, o=q, z=lse: PG.attn_paged_prefill(sh, q, gate, cu, st, kp, vp, tcu, ids, o, z, ws)  # noqa: E731
    weigh = lambda q=q, z=lse, kp=k, wi=w, wo=w: PG.attn_key_weights(sh, q, z, cu, st, kp, tcu, ids, 1.0, wi, wo, ws)  # noqa: E731
    evict = lambda kp=k, vp=v, w=w, i=torch.zeros(99, dtype=torch.int32): PG.attn_evict(sh, [5, 24], [4, 9], [1, 1], [1, 1], kp, vp, w, tcu, ids, [0, 1, 2], [1, 2], i, ws)  # noqa: E731
    for call in (append, attend, weigh, evict):
        refused(call, -9)                                                     # nothing else is wrong: the workspace is too small
    for bad in (turned, wide):
        for name in ("q", "k_", "v_", "out"):
            refused(append, -3, *[bad(x) if n == name else x for n, x in (("q", q), ("k_", kv), ("v_", kv))], k, v, bad(q) if name == "out" else q)
        for pools in ((bad(k), v), (k, bad(v)), (bad(k), bad(v))):
            refused(lambda: append(kp=pools[0], vp=pools[1]), -3)
            refused(lambda: attend(kp=pools[0], vp=pools[1]), -3)
            refused(lambda: evict(kp=pools[0], vp=pools[1]), -3)
        refused(lambda: weigh(kp=bad(k)), -3)
        for kw in (dict(q=bad(q)), dict(gate=bad(q)), dict(o=bad(q)), dict(z=wide(lse))):
            refused(lambda: attend(**kw), -3)
        for kw in (dict(q=bad(q)), dict(z=wide(lse)), dict(wi=bad(w)), dict(wo=bad(w), wi=None)):
            refused(lambda: weigh(**kw), -3)
        refused(lambda: evict(w=bad(w)), -3)
    refused(lambda: evict(i=torch.zeros(198, dtype=torch.int32)[::2]), -3)
    for w_ in (w[:39], w[:, :1], torch.zeros(40, 2, 32)):                     # fewer weights than the keys' pages have rows
        refused(lambda: weigh(wi=None, wo=w_), -3)
        refused(lambda: evict(w=w_), -3)
    refused(lambda: attend(kp=torch.zeros(40, 3, 16, 64)[:, :, :, :], vp=torch.zeros(40, 3, 16, 64)), -3)


def test_the_token_stride_of_one_token_is_nobodys(no_stream):
    import torch
    a = torch.zeros(4, 1, 64).transpose(0, 1)                                 # [1][4][64] with a token stride of 64
    assert a.stride(0) == 64 and PG._ld(a) == 256 and PG._ld(a[:, :2]) == 128
    assert PG._ld(torch.zeros(9, 12, 64)[:, 4:8]) == 768 and PG._ld(torch.zeros(1, 256)) == 256 and PG._ld(torch.zeros(0, 4, 64)) == 256


# ----------------------------------------------------------------------------- GPU
def f64(bits):
    return wl.to_f32(bits).astype(np.float64)


class Paged:
    """A call's pools on the device: every request's pages in no order, whatever no request holds NaN."""

    def __init__(self, seed, H_q, H_kv, d, P, lens, starts, shared=0, extra=0, stride_pad=0):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.H_q, self.H_kv, self.d, self.P = H_q, H_kv, d, P
        self.lens, self.starts = list(lens), list(starts)
        self.total = [s + n for s, n in zip(starts, lens)]
        self.T, R = sum(lens), len(lens)
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        sp = shared // P
        pages = [-(-t // P) for t in self.total]
        assert all(s >= sp * P for s in starts)
        n_pages = sp + sum(p - sp for p in pages) + extra + 2
        ids = rng.permutation(n_pages).astype(np.int32)
        common, rest = ids[:sp], list(ids[sp:])
        self.table = [np.concatenate([common, [rest.pop() for _ in range(p - sp)]]).astype(np.int32) for p in pages]
        self.spare = np.array(rest, np.int32)
        self.page_cu = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.page_ids = np.concatenate(self.table + [np.zeros(0, np.int32)]).astype(np.int32)
        size = H_kv * P * d
        self.k_np = np.full((n_pages, size + stride_pad), 0x7fc0, np.uint16)
        self.v_np = np.full((n_pages, size + stride_pad), np.nan, np.float16)
        self.k_rows, self.v_rows = [], []
        for r, t in enumerate(self.total):
            k = wl.f32_to_bf16_bits(rng.standard_normal((t, H_kv, d), dtype=np.float32))
            v = rng.standard_normal((t, H_kv, d)).astype(np.float16)
            if r > 0:
                k[:sp * P], v[:sp * P] = self.k_rows[0][:sp * P], self.v_rows[0][:sp * P]
            self.k_rows.append(k)
            self.v_rows.append(v)
        self.shape = AT.make_attn_shape(H_q, H_kv, d, "bf16")
        self.torch = torch

    def place(self, r, count, table=None):
        j = np.arange(count)
        return (table if table is not None else self.table[r])[j // self.P], j % self.P

    def view(self, a, d=None):
        return a[:, :self.H_kv * self.P * (d or self.d)].reshape(a.shape[0], self.H_kv, self.P, -1)

    def fill(self, held_only=False):
        """Rows into the pools (those held before the call only, or all) and the pools to the device."""
        for r in range(len(self.lens)):
            n = self.starts[r] if held_only else self.total[r]
            page, row = self.place(r, n)
            self.view(self.k_np)[page, :, row] = self.k_rows[r][:n]
            self.view(self.v_np)[page, :, row] = self.v_rows[r][:n]
        return self.fill_values()

    def fill_values(self):
        """The pools as they are to the device."""
        t = self.torch
        self.k_dev = t.from_numpy(self.k_np.view(np.int16)).cuda().view(t.bfloat16)
        self.v_dev = t.from_numpy(self.v_np).cuda()
        size = self.H_kv * self.P * self.d
        self.k_pool, self.v_pool = (x[:, :size].unflatten(1, (self.H_kv, self.P, self.d)) for x in (self.k_dev, self.v_dev))
        return self

    def workspace(self, tokens=None, ids=None):
        t = self.torch
        n = PG.attn_paged_workspace_bytes(self.shape, len(self.lens), self.T if tokens is None else tokens, self.page_ids.size if ids is None else ids)
        return t.full((n,), 0xA5, dtype=t.uint8, device="cuda")

    def bf16(self, *shape, s=1.0):
        return wl.f32_to_bf16_bits((self.rng.standard_normal(shape, dtype=np.float32) * np.float32(s)).astype(np.float32))

    def dev(self, bits):
        return self.torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(self.torch.bfloat16)


def bits_of(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def logit_error(c, q):
    """A bound of the error of a scaled logit in fp32."""
    worst = max([np.sqrt((f64(k) ** 2).sum(-1)).max() for k in c.k_rows if k.size] + [0.0]) * np.sqrt((f64(q) ** 2).sum(-1)).max()
    return (c.d + 16) * 2.0 ** -24 * c.d ** -0.5 * worst


ROPE = [  # H_q, H_kv, d, P, rot, layout, dtype, lens, starts, pos
    (4, 2, 64, 16, 64, "half", "bf16", [1], [0], [0]),
    (4, 2, 64, 16, 64, "interleaved", "bf16", [5, 0, 37], [15, 3, 16], [7, 0, 2000000000]),
    (6, 2, 128, 32, 32, "half", "f32", [33, 1], [31, 0], None),
    (8, 1, 256, 64, 48, "interleaved", "f32", [3, 70], [1, 62], [123456789, 1]),
    (3, 3, 128, 16, 0, "half", "bf16", [17], [8], [3]),
    (16, 2, 128, 128, 128, "half", "bf16", [1] * 70, list(range(100, 170)), None),
    (4, 4, 64, 16, 16, "half", "bf16", [1100], [5], [900000]),
    (2, 1, 256, 32, 256, "half", "bf16", [9001], [0], [0]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,rot,layout,dtype,lens,starts,pos", ROPE)
@pytest.mark.parametrize("packed", [True, False])
def test_rope_append(H_q, H_kv, d, P, rot, layout, dtype, lens, starts, pos, packed):
    import torch
    c = Paged(5, H_q, H_kv, d, P, lens, starts, stride_pad=0 if packed else 24).fill(held_only=True)
    freqs, amp = PG.attn_rope_freqs(rot, 10000.0, "ramp", 8.0, 4096.0) if rot else (np.zeros(0), 1.0)
    rope = PG.make_attn_rope(freqs, layout, amp, dtype)
    heads = [H_q, H_kv, H_kv]
    x = torch.randn(c.T, sum(heads) * d + (0 if packed else 8), generator=torch.Generator().manual_seed(1))
    x = x if dtype == "f32" else x.bfloat16()
    ref = x.double().numpy()
    if packed:                       # tensors of their own, or column ranges of one projection's output
        parts = [y.contiguous().cuda().unflatten(1, (-1, d)) for y in x.split([h * d for h in heads], 1)]
    else:
        parts = [y.unflatten(1, (-1, d)) for y in x.cuda()[:, 8:].split([h * d for h in heads], 1)]
        ref = ref[:, 8:]
    q, k, v = (y.reshape(c.T, -1, d) for y in np.split(ref, np.cumsum([h * d for h in heads])[:2], 1))
    q_out = parts[0] if packed and dtype == "bf16" else torch.zeros(c.T, H_q, d, dtype=torch.bfloat16, device="cuda")   # in place where it may be
    before_k, before_v = c.k_dev.clone(), c.v_dev.clone()
    PG.attn_rope_append(c.shape, rope, *parts, c.cu, pos, starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids, q_out, c.workspace())
    got_q = q_out.double().cpu().numpy()
    k_after, v_after = c.k_pool.double().cpu().numpy(), bits_of(c.v_pool)
    m = rot // 2
    for r, n in enumerate(lens):
        if n == 0:
            continue
        s, p0 = slice(c.cu[r], c.cu[r + 1]), starts[r] if pos is None else pos[r]
        page, row = c.place(r, c.total[r])
        page, row = page[starts[r]:], row[starts[r]:]
        few = np.unique(np.r_[0:min(n, 20), max(0, n - 20):n, n // 2])     # of long calls some tokens
        for got, src in ((got_q[s], q[s]), (k_after[page, :, row], k[s])):
            for i in few:
                want = po.rotate(src[i:i + 1], p0 + i, freqs, layout, amp)
                pair = np.abs(src[i:i + 1]).copy()
                if m:
                    a, b = (slice(0, m), slice(m, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
                    both = pair[..., a] + pair[..., b]
                    pair[..., a], pair[..., b] = both, both
                assert (np.abs(got[i:i + 1] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * amp * pair).all(), (r, i)
        assert np.array_equal(v_after[page, :, row], v[s].astype(np.float32).astype(np.float16).view(np.uint16)), r
    # nothing else was written
    mask = torch.ones_like(c.k_dev, dtype=torch.bool)
    mv = mask[:, :H_kv * P * d].unflatten(1, (H_kv, P, d))
    for r in range(len(lens)):
        page, row = c.place(r, c.total[r])
        mv[torch.from_numpy(page[starts[r]:].astype(np.int64)).cuda(), :, torch.from_numpy(row[starts[r]:]).cuda()] = False
    for a, b in ((before_k, c.k_dev), (before_v, c.v_dev)):
        assert torch.equal(a.view(torch.int16)[mask], b.view(torch.int16)[mask])


ATTEND = [  # H_q, H_kv, d, P, lens, starts, shared, gate, dtype
    (4, 2, 64, 16, [1], [0], 0, False, "bf16"),                              # one token, one row
    (4, 2, 128, 16, [1, 0, 2, 17, 64, 65], [0, 7, 1, 15, 33, 200], 0, True, "f32"),
    (8, 1, 256, 32, [3, 130], [31, 40], 0, False, "bf16"),
    (6, 2, 64, 64, [5, 200], [100, 63], 0, False, "bf16"),                   # a group of three: not packed
    (1, 1, 128, 128, [129], [0], 0, False, "f32"),
    (16, 2, 128, 256, [300, 40], [700, 0], 0, True, "bf16"),
    (16, 2, 128, 16, [1, 1, 1], [1500, 1023, 2047], 0, False, "bf16"),       # decoding: the few-rows kernel, walks cut
    (8, 8, 64, 32, [2, 1], [1100, 5000], 0, True, "f32"),
    (8, 1, 256, 16, [1, 2], [1300, 1022], 0, False, "bf16"),
    (4, 1, 128, 64, [1] * 40, [1000 + 37 * i for i in range(40)], 0, False, "bf16"),
    (16, 2, 128, 64, [1, 1, 100], [4000, 1200, 900], 0, False, "bf16"),      # both kinds in one call
    (16, 2, 128, 16, [1, 30, 200], [600, 512, 700], 512, False, "bf16"),     # a shared prefix
    (32, 4, 128, 128, [700], [2000], 0, False, "bf16"),                      # walks cut, two heads to a workgroup
    (2, 2, 256, 128, [50], [9000], 0, False, "f32"),
    (16, 2, 64, 16, [1], [20000], 0, False, "f32"),                          # more steps than page ids are held at once
    (4, 2, 128, 16, [600], [8000], 0, False, "bf16"),
]


def run_attend(c, q, gate, dtype, lse=True, stream=None):
    t = c.torch
    sh = AT.make_attn_shape(c.H_q, c.H_kv, c.d, dtype)
    o = t.full((c.T, c.H_q, c.d), float("nan"), dtype=t.float32 if dtype == "f32" else t.bfloat16, device="cuda")
    z = t.full((c.T, c.H_q), float("nan"), device="cuda") if lse else None
    PG.attn_paged_prefill(sh, c.dev(q), c.dev(gate) if gate is not None else None, c.cu, c.starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids, o, z,
                          c.workspace(), stream)
    return o, z


def check_attend(c, q, gate, dtype, o, z):
    scale = c.d ** -0.5
    o, z = o.double().cpu().numpy(), z.cpu().numpy().astype(np.float64) if z is not None else None
    le = logit_error(c, q) if c.T else 0.0
    for r in range(len(c.lens)):
        if c.lens[r] == 0:
            continue
        s = slice(c.cu[r], c.cu[r + 1])
        k, v = f64(c.k_rows[r]), c.v_rows[r].astype(np.float64)
        ref = ao.attention_suffix(f64(q[s]), k, v, c.starts[r], scale)
        if gate is not None:
            ref = ao.output_gate(ref, f64(gate[s]))
        tol = 2.0 ** -8 * np.abs(v).max() + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
        assert (np.abs(o[s] - ref) <= tol).all(), (r, np.nanmax(np.abs(o[s] - ref)), np.isnan(o[s]).sum())
        if z is not None:
            zr = po.row_lse(f64(q[s]), k, c.starts[r], scale)
            assert (np.abs(z[s] - zr) <= le + 2.0 ** -20 * (1 + np.abs(zr))).all(), (r, np.nanmax(np.abs(z[s] - zr)))


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts,shared,gate,dtype", ATTEND)
def test_paged_prefill(H_q, H_kv, d, P, lens, starts, shared, gate, dtype):
    c = Paged(11, H_q, H_kv, d, P, lens, starts, shared, stride_pad=8).fill()
    q, g = c.bf16(c.T, H_q, d, s=2.0), c.bf16(c.T, H_q, d) if gate else None
    o, z = run_attend(c, q, g, dtype)
    check_attend(c, q, g, dtype, o, z)
    o2, _ = run_attend(c, q, g, dtype, lse=False)
    assert np.array_equal(bits_of(o2), bits_of(o))                          # asking for lse changes no bit of o


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_paged_prefill_equals_the_slot_form_bit_for_bit(seed):
    """The same rows in slots and in pages: the same kernels walk them in the same order."""
    import torch
    rng = np.random.default_rng(100 + seed)
    H_q, H_kv = [(16, 2), (4, 4), (8, 1), (32, 4), (6, 2), (16, 2)][seed]
    d, P = int(rng.choice([64, 128, 256])), int(rng.choice([16, 64, 128]))
    R = int(rng.integers(1, 6))
    lens, starts = [int(x) for x in rng.integers(1, 300, R)], [int(x) for x in rng.integers(0, 2500, R)]
    if seed % 2:
        lens = [1] * R
    c = Paged(200 + seed, H_q, H_kv, d, P, lens, starts).fill()
    q = c.bf16(c.T, H_q, d)
    cap = max(c.total)
    kc, vc = np.zeros((R, cap, H_kv, d), np.uint16), np.zeros((R, cap, H_kv, d), np.float16)
    # the slot form appends itself: its new values come in bf16, so the pages get what that widens to
    v_new = [wl.f32_to_bf16_bits(v[s:].astype(np.float32)) for v, s in zip(c.v_rows, starts)]
    for r in range(R):
        c.v_rows[r][starts[r]:] = wl.to_f32(v_new[r]).astype(np.float16)
        kc[r, :starts[r]], vc[r, :starts[r]] = c.k_rows[r][:starts[r]], c.v_rows[r][:starts[r]]
    c.fill()
    o, z = run_attend(c, q, None, "f32")
    check_attend(c, q, None, "f32", o, z)
    sh = AT.make_attn_shape(H_q, H_kv, d, "f32")
    os_ = torch.zeros_like(o)
    ws = torch.empty(AT.attn_workspace_bytes(sh, R, c.T), dtype=torch.uint8, device="cuda")
    AT.attn_tune_split(False)                                               # whole walks (the paged form's small calls cut more of them)
    try:
        o, _ = run_attend(c, q, None, "f32", lse=False)
        AT.attn_suffix_prefill(sh, c.dev(q), c.dev(np.concatenate([k[s:] for k, s in zip(c.k_rows, starts)])), c.dev(np.concatenate(v_new)), None, c.cu, starts,
                               c.dev(kc), torch.from_numpy(vc).cuda(), list(range(R)), os_, ws)
    finally:
        AT.attn_tune_split(True)
    assert torch.equal(o, os_)


WEIGHTS = [  # H_q, H_kv, d, P, lens, starts, w_in: None, "in", "same"
    (4, 2, 64, 16, [1], [0], None),
    (4, 2, 128, 16, [1, 0, 0, 2, 33], [0, 70, 0, 300, 15], "in"),
    (8, 1, 256, 32, [3, 130], [31, 400], "same"),
    (6, 2, 64, 64, [5, 200], [100, 63], "in"),
    (16, 2, 128, 256, [300, 40], [700, 0], "in"),
    (32, 1, 128, 16, [1, 1, 1], [1500, 1023, 255], "in"),
    (48, 1, 64, 128, [2], [600], None),
    (16, 2, 128, 64, [1200], [0], "same"),                                  # rows cut into parts
    (3, 3, 256, 16, [900, 7], [33, 500], "in"),
    (16, 4, 128, 32, [1] * 70, [10 * i for i in range(70)], "in"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts,w_in", WEIGHTS)
def test_key_weights(H_q, H_kv, d, P, lens, starts, w_in):
    import torch
    c = Paged(21, H_q, H_kv, d, P, lens, starts).fill()
    q = c.bf16(c.T, H_q, d, s=2.0)
    scale, decay = d ** -0.5, 0.75
    lse = np.zeros((c.T, H_q), np.float32)
    for r in range(len(lens)):
        if lens[r]:
            lse[c.cu[r]:c.cu[r + 1]] = po.row_lse(f64(q[c.cu[r]:c.cu[r + 1]]), f64(c.k_rows[r]), starts[r], scale)
    n_pages = c.k_np.shape[0]
    w_np = np.full((n_pages, H_kv, P), np.nan, np.float32)
    held = [c.rng.exponential(size=(s, H_kv)).astype(np.float32) for s in starts]
    for r, s in enumerate(starts):
        page, row = c.place(r, s)
        w_np[page, :, row] = held[r]
    w0 = torch.from_numpy(w_np).cuda()
    w_out = w0 if w_in == "same" else torch.full_like(w0, float("nan"))
    PG.attn_key_weights(c.shape, c.dev(q), torch.from_numpy(lse).cuda(), c.cu, starts, c.k_pool, c.page_cu, c.page_ids, decay,
                        None if w_in is None else w0, w_out, c.workspace())
    got = w_out.cpu().numpy().astype(np.float64)
    untouched = np.ones(got.shape, bool)
    rtol = np.expm1(logit_error(c, q) + 2.0 ** -22 * (1 + np.abs(lse).max())) + (max(lens) * (H_q // H_kv) + 8) * 2.0 ** -24
    for r in range(len(lens)):
        page, row = c.place(r, c.total[r])
        s = slice(c.cu[r], c.cu[r + 1])
        ref = po.key_weights(f64(q[s]), lse[s], f64(c.k_rows[r]), starts[r], scale, decay, held[r] if w_in else None) if lens[r] else \
            (decay * held[r].astype(np.float64) if w_in else np.zeros((starts[r], H_kv)))
        x = got[page, :, row]
        assert (np.abs(x - ref) <= rtol * ref).all(), (r, np.nanmax(np.abs(x - ref) / ref))
        untouched[page, :, row] = False
    assert np.isnan(got[untouched]).all()


EVICT = [  # H_kv, d, P, rows, keep, first, recent, weights
    (2, 64, 16, [40], [10], [2], [3], "normal"),
    (1, 128, 16, [1, 0, 33, 16], [1, 5, 16, 16], [0, 0, 4, 0], [0, 0, 4, 16], "normal"),
    (2, 64, 32, [100, 70], [100, 90], [0, 5], [0, 5], "normal"),              # everything is kept
    (4, 256, 64, [1000, 31], [500, 31], [4, 0], [64, 0], "ties"),
    (2, 64, 16, [300], [100], [0], [0], "equal"),
    (2, 128, 128, [5000], [1234], [4], [64], "odd"),                          # NaN, infinities, zeros of both signs, negative ones
    (1, 64, 16, [50], [30], [10], [20], "normal"),                            # first and last rows alone
    (3, 64, 256, [20000, 9, 4097], [2000, 3, 4096], [4, 1, 0], [128, 1, 0], "ties"),
    (2, 64, 16, [64], [0], [0], [0], "normal"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("H_kv,d,P,rows,keep,first,recent,kind", EVICT)
def test_evict(H_kv, d, P, rows, keep, first, recent, kind):
    import torch
    kept = [min(a, b) for a, b in zip(keep, rows)]
    new_n = [-(-m // P) for m in kept]
    c = Paged(31, H_kv, H_kv, d, P, [0] * len(rows), rows, extra=sum(new_n)).fill()
    w_np = np.full(c.k_np.shape[:1] + (H_kv, P), np.nan, np.float32)
    w_rows = []
    for r, n in enumerate(rows):
        w = c.rng.standard_normal((n, H_kv)).astype(np.float32)
        if kind == "ties":
            w = np.round(w)
        if kind == "equal":
            w[:] = 0.25
        if kind == "odd":
            w = np.maximum(w, 0)                                             # the lowest row of many equal ones
            for x in (np.nan, np.inf, -np.inf, -0.0, 0.0, -1.0, 1e-45):
                w[c.rng.integers(0, n, 300), :] = x
        w_rows.append(w)
        page, row = c.place(r, n)
        w_np[page, :, row] = w
    spare = list(c.spare)
    new_table = [np.array([spare.pop() for _ in range(m)], np.int32) for m in new_n]
    new_cu = np.concatenate([[0], np.cumsum(new_n)]).astype(np.int32)
    w_pool = torch.from_numpy(w_np).cuda()
    index = torch.full((max(1, sum(kept) * H_kv),), -7, dtype=torch.int32, device="cuda")
    PG.attn_evict(c.shape, rows, keep, first, recent, c.k_pool, c.v_pool, w_pool, c.page_cu, c.page_ids, new_cu,
                  np.concatenate(new_table + [np.zeros(0, np.int32)]), index, c.workspace(0, c.page_ids.size + sum(new_n)))
    k_got, v_got, w_got, idx = bits_of(c.k_pool), bits_of(c.v_pool), w_pool.cpu().numpy(), index.cpu().numpy()
    k_ref, v_ref, w_ref = c.view(c.k_np).copy(), c.view(c.v_np).copy(), w_np.copy()
    at = 0
    for r in range(len(rows)):
        page, row = c.place(r, kept[r], new_table[r])
        for g in range(H_kv):
            want = po.rows_kept(w_rows[r][:, g], keep[r], first[r], recent[r])
            assert len(want) == kept[r]
            assert np.array_equal(idx[at:at + kept[r]], want), (r, g)
            at += kept[r]
            k_ref[page, g, row] = c.k_rows[r][want, g]
            v_ref[page, g, row] = c.v_rows[r][want, g]
            w_ref[page, g, row] = w_rows[r][want, g]
    assert np.array_equal(k_got, k_ref) and np.array_equal(v_got, v_ref.view(np.uint16))
    assert np.array_equal(w_got.view(np.uint32), w_ref.view(np.uint32))


@pytest.mark.gpu
def test_pages_behind_32_bit_offsets():
    """Pages whose offsets pass 2^31 elements (2^32 bytes and more): every operator reads and writes the right ones."""
    import torch
    H_q, H_kv, d, P, stride = 4, 2, 64, 16, 1 << 31
    c = Paged(41, H_q, H_kv, d, P, [9], [30], extra=1)
    base_k, base_v = (torch.empty(3 * stride + H_kv * P * d, dtype=x, device="cuda") for x in (torch.bfloat16, torch.float16))
    shape, strides = (4, H_kv, P, d), (stride, P * d, d, 1)
    c.k_pool, c.v_pool = base_k.as_strided(shape, strides), base_v.as_strided(shape, strides)
    w_pool = torch.empty(3 * stride + H_kv * P, device="cuda").as_strided((4, H_kv, P), (stride, P, 1))
    c.table, c.page_ids = [np.array([3, 1, 2], np.int32)], np.array([3, 1, 2], np.int32)
    for x in (c.k_pool, c.v_pool, w_pool):
        x.fill_(float("nan"))
    page, row = (torch.from_numpy(x.astype(np.int64)).cuda() for x in c.place(0, 39))
    k, v = c.dev(c.k_rows[0]), torch.from_numpy(c.v_rows[0]).cuda()
    c.k_pool[page[:30], :, row[:30]], c.v_pool[page[:30], :, row[:30]] = k[:30], v[:30]
    q = c.bf16(9, H_q, d)
    c.v_rows[0][30:] = c.v_rows[0][30:].astype(np.float32).astype(np.float16)
    v_new = c.dev(wl.f32_to_bf16_bits(c.v_rows[0][30:].astype(np.float32)))
    c.v_rows[0][30:] = v_new.float().cpu().numpy().astype(np.float16)
    q_out = torch.zeros(9, H_q, d, dtype=torch.bfloat16, device="cuda")
    PG.attn_rope_append(c.shape, PG.make_attn_rope([]), c.dev(q), k[30:].contiguous(), v_new, c.cu, None, c.starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids,
                        q_out, c.workspace())
    assert np.array_equal(bits_of(q_out), q) and torch.equal(c.k_pool[page, :, row], k)
    o, z = run_attend(c, q, None, "f32")
    check_attend(c, q, None, "f32", o, z)
    PG.attn_key_weights(c.shape, q_out, z, c.cu, c.starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w_pool, c.workspace())
    w = w_pool[page, :, row].cpu().numpy()
    assert abs(w.sum() - 9 * H_q) <= 1e-4 * 9 * H_q
    index = torch.zeros(16 * H_kv, dtype=torch.int32, device="cuda")
    PG.attn_evict(c.shape, [39], [16], [1], [4], c.k_pool, c.v_pool, w_pool, c.page_cu, c.page_ids, [0, 1], [0], index, c.workspace(0, 4))
    idx = index.cpu().numpy().reshape(H_kv, 16)
    for g in range(H_kv):
        assert list(idx[g]) == po.rows_kept(w[:, g], 16, 1, 4)
        assert torch.equal(c.k_pool[0, g], k[torch.from_numpy(idx[g].astype(np.int64)).cuda(), g])


@pytest.mark.gpu
def test_calls_on_another_stream_and_again_give_the_same_bits():
    import torch
    c = Paged(51, 16, 2, 128, 64, [1, 40, 1], [3000, 800, 5000]).fill()
    q = c.bf16(c.T, 16, 128)
    o, z = run_attend(c, q, None, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2, z2 = run_attend(c, q, None, "bf16")
        w = torch.zeros(c.k_np.shape[0], 2, 64, device="cuda")
        PG.attn_key_weights(c.shape, c.dev(q), z2, c.cu, c.starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w, c.workspace())
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(z, z2)
    w2 = torch.zeros_like(w)
    PG.attn_key_weights(c.shape, c.dev(q), z, c.cu, c.starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w2, c.workspace())
    assert torch.equal(w, w2)


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts,at", [
    (4, 2, 64, 16, [40], [3], 20),                    # inside one tile
    (16, 2, 128, 32, [24, 5], [100, 60], 2),          # packed rows
    (4, 1, 128, 16, [3], [1300], 1),                  # the few-rows kernel, walks cut
    (8, 8, 256, 64, [70], [2500], 33),                # walks cut, parts that see nothing
    (16, 2, 128, 64, [400], [600], 250),              # two heads to a workgroup or one
    (1, 1, 64, 16, [9], [1100], 4),
])
@pytest.mark.parametrize("what", [np.inf, np.nan])
def test_what_a_later_token_holds_does_not_reach_earlier_rows(H_q, H_kv, d, P, lens, starts, at, what):
    """Token `at` of every request has a value row that is not finite and a key of NaN: the rows before it are those of a request that
    ends there, the rows from it on are not finite."""
    c = Paged(61, H_q, H_kv, d, P, lens, starts)
    for r in range(len(lens)):
        c.v_rows[r][starts[r] + at] = what
        c.k_rows[r][starts[r] + at] = 0x7fc0
    c.fill()
    q = c.bf16(c.T, H_q, d)
    o, z = run_attend(c, q, None, "f32")
    o, z = o.double().cpu().numpy(), z.double().cpu().numpy()
    for r in range(len(lens)):
        cut, s0 = starts[r] + at, c.cu[r]
        k, v = f64(c.k_rows[r][:cut]), c.v_rows[r][:cut].astype(np.float64)
        ref = ao.attention_suffix(f64(q[s0:s0 + at]), k, v, starts[r], d ** -0.5)
        assert (np.abs(o[s0:s0 + at] - ref) <= 2.0 ** -8 * np.abs(v).max()).all(), r
        zr = po.row_lse(f64(q[s0:s0 + at]), k, starts[r], d ** -0.5)
        bound = (d + 16) * 2.0 ** -24 * d ** -0.5 * np.sqrt((k ** 2).sum(-1)).max() * np.sqrt((f64(q) ** 2).sum(-1)).max()
        assert (np.abs(z[s0:s0 + at] - zr) <= bound + 2.0 ** -20 * (1 + np.abs(zr))).all()
        assert not np.isfinite(o[s0 + at:s0 + lens[r]]).any()


@pytest.mark.gpu
def test_key_weights_of_rows_and_keys_that_are_not_numbers_stay_theirs():
    """A key of NaN has a weight of NaN and no other has; a query row of NaN reaches the keys that it sees and no others."""
    import torch
    c = Paged(62, 4, 2, 128, 16, [40, 1], [300, 20])
    c.k_rows[0][310, 1] = 0x7fc0
    c.fill()
    q = c.bf16(41, 4, 128)
    q[10, 1] = 0x7fc0                                  # token 10 of the first request, head group 0
    lse = torch.zeros(41, 4, device="cuda") + 8.0
    w = torch.full((c.k_np.shape[0], 2, 16), 7.0, device="cuda")
    PG.attn_key_weights(c.shape, c.dev(q), lse, c.cu, c.starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w, c.workspace())
    w = w.cpu().numpy()
    page, row = c.place(0, 340)
    got = w[page, :, row]
    assert np.isnan(got[:311, 0]).all() and np.isfinite(got[311:, 0]).all()
    assert np.isnan(got[310, 1]) and np.isfinite(np.delete(got[:, 1], 310)).all()
    page, row = c.place(1, 21)
    assert np.isfinite(w[page, :, row]).all()


@pytest.mark.gpu
def test_a_session_of_prompts_decoding_and_eviction_matches_the_oracle():
    """The operators in turn, as a serving program runs them: after an eviction the requests go on with fewer rows and the same positions."""
    import torch
    from paper_2605_05219_amd.paged_session import PagedLayer
    H_q, H_kv, d, R = 4, 2, 64, 2
    layer = PagedLayer(H_q, H_kv, d, R, 40, page_rows=16, decay=0.9)
    freqs = po.rope_freqs(d)[0]
    gen = torch.Generator().manual_seed(3)
    held = [dict(k=np.zeros((0, H_kv, d)), v=np.zeros((0, H_kv, d)), w=np.zeros((0, H_kv))) for _ in range(R)]
    pos = [0, 0]
    for lens in ([70, 33], [1, 1], [5, 0], [1, 1]):
        q, k, v = (torch.randn(sum(lens), h, d, generator=gen).bfloat16() for h in (H_q, H_kv, H_kv))
        o = layer.step(q.cuda(), k.cuda(), v.cuda(), lens).double().cpu().numpy()
        at = 0
        for r, n in enumerate(lens):
            if n == 0:
                held[r]["w"] = held[r]["w"] * 0.9
                continue
            s = slice(at, at + n)
            at += n
            bf = lambda x: torch.from_numpy(x).bfloat16().double().numpy()  # noqa: E731
            qr, kr = (bf(po.rotate(x[s].double().numpy(), pos[r], freqs, "half", 1.0)) for x in (q, k))
            h, c = held[r], held[r]["k"].shape[0]
            h["k"], h["v"] = np.concatenate([h["k"], kr]), np.concatenate([h["v"], v[s].double().numpy()])
            ref = ao.attention_suffix(qr, h["k"], h["v"], c, d ** -0.5)
            # a rotated value may round the other way: 2^-7 of q and of k moves a logit by 2^-6 |q||k| scale at the very most, where it is far less
            assert np.abs(o[s] - ref).max() <= 2.0 ** -5 * np.abs(h["v"]).max()
            h["w"] = po.key_weights(qr, po.row_lse(qr, h["k"], c, d ** -0.5), h["k"], c, d ** -0.5, 0.9, h["w"])
            pos[r] += n
        if layer.rows.max() > 60:
            before, w_pool = [list(p) for p in layer.pages], layer.w_pool.cpu().numpy()
            rows = layer.rows.copy()
            layer.evict(60, 40, first=2, recent=8)
            for r in range(R):
                if rows[r] <= 60:
                    continue
                j = np.arange(rows[r])
                w = w_pool[np.asarray(before[r])[j // 16], :, j % 16]
                assert np.allclose(w, held[r]["w"], rtol=2e-2, atol=1e-3)
                idx = [po.rows_kept(w[:, g], 40, 2, 8) for g in range(H_kv)]
                for x in held[r]:
                    held[r][x] = np.stack([held[r][x][idx[g], g] for g in range(H_kv)], axis=1)
                assert layer.rows[r] == 40 and len(layer.pages[r]) == 3 and layer.pos[r] == pos[r]
    assert len(layer.free) + sum(len(p) for p in layer.pages) == 40


@pytest.mark.gpu
def test_many_calls_with_long_page_tables_in_a_row_keep_their_own_plans():
    """More calls than there are staging buffers, none waited for, each with page tables of its own (and all too long for the arguments)."""
    import torch
    rng = np.random.default_rng(7)
    c = Paged(71, 4, 2, 64, 16, [1] * 24, [int(x) for x in rng.integers(1200, 2400, 24)]).fill()
    assert c.page_ids.size > 1792
    q = c.bf16(c.T, 4, 64)
    want, wz = run_attend(c, q, None, "f32")
    torch.cuda.synchronize()
    qd, ws = c.dev(q), c.workspace()
    sh = AT.make_attn_shape(4, 2, 64, "f32")
    outs = []
    for i in range(30):                     # the requests in another order every time
        order = rng.permutation(24)
        cu = np.arange(25, dtype=np.int32)
        tables = [c.table[r] for r in order]
        tcu = np.concatenate([[0], np.cumsum([t.size for t in tables])]).astype(np.int32)
        o, z = torch.zeros(24, 4, 64, device="cuda"), torch.zeros(24, 4, device="cuda")
        at = torch.from_numpy(order).cuda()
        w = torch.zeros(c.k_np.shape[0], 2, 16, device="cuda") if i % 3 == 0 else None
        PG.attn_paged_prefill(sh, qd[at].contiguous(), None, cu, np.asarray(c.starts)[order], c.k_pool, c.v_pool, tcu, np.concatenate(tables), o, z, ws)
        if w is not None:
            PG.attn_key_weights(sh, qd[at].contiguous(), z, cu, np.asarray(c.starts)[order], c.k_pool, tcu, np.concatenate(tables), 1.0, None, w, ws)
        outs.append((at, o, z, w))
    torch.cuda.synchronize()
    for at, o, z, w in outs:
        assert torch.equal(o, want[at]) and torch.equal(z, wz[at])
        if w is not None:                   # every row of queries spreads a weight of one over its request's rows
            page, row = c.place(3, c.total[3])
            assert abs(float(w[torch.from_numpy(page.astype(np.int64)).cuda(), :, torch.from_numpy(row).cuda()].sum()) - 4) <= 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(8))
def test_random_calls_of_the_weights_and_the_eviction_that_follows(seed):
    """Ragged batches of both kinds of requests, against the oracle, and an eviction by the weights that came out."""
    import torch
    rng = np.random.default_rng(900 + seed)
    H_q, H_kv = [(16, 2), (8, 8), (6, 2), (32, 4), (8, 1), (4, 4), (20, 4), (16, 4)][seed]
    d, P, R = int(rng.choice([64, 128, 256])), int(rng.choice([16, 32, 128, 256])), int(rng.integers(2, 7))
    lens = [int(x) for x in rng.choice([0, 1, 2, 63, 64, 65, 300, 700], R)]
    starts = [int(x) for x in rng.integers(0, 2000, R)]
    lens[0] = max(lens[0], 1)
    kept = [min(s + n, int(rng.integers(1, 600))) for s, n in zip(starts, lens)]
    new_n = [-(-m // P) for m in kept]
    c = Paged(950 + seed, H_q, H_kv, d, P, lens, starts, extra=sum(new_n)).fill()
    q = c.bf16(c.T, H_q, d, s=1.5)
    lse = np.zeros((c.T, H_q), np.float32)
    for r in range(R):
        if lens[r]:
            lse[c.cu[r]:c.cu[r + 1]] = po.row_lse(f64(q[c.cu[r]:c.cu[r + 1]]), f64(c.k_rows[r]), starts[r], d ** -0.5)
    w = torch.full((c.k_np.shape[0], H_kv, P), float("nan"), device="cuda")
    ws = c.workspace(ids=c.page_ids.size + sum(new_n))
    PG.attn_key_weights(c.shape, c.dev(q), torch.from_numpy(lse).cuda(), c.cu, starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w, ws)
    got = w.cpu().numpy()
    rtol = np.expm1(logit_error(c, q) + 2.0 ** -22 * (1 + np.abs(lse).max())) + (max(lens) * (H_q // H_kv) + 8) * 2.0 ** -24
    spare = list(c.spare)
    new_table = [np.array([spare.pop() for _ in range(m)], np.int32) for m in new_n]
    new_cu = np.concatenate([[0], np.cumsum(new_n)]).astype(np.int32)
    index = torch.zeros(max(1, sum(kept) * H_kv), dtype=torch.int32, device="cuda")
    first, recent = [min(2, m) for m in kept], [min(5, max(0, m - 2)) for m in kept]
    PG.attn_evict(c.shape, c.total, kept, first, recent, c.k_pool, c.v_pool, w, c.page_cu, c.page_ids, new_cu,
                  np.concatenate(new_table + [np.zeros(0, np.int32)]), index, ws)
    idx, k_got, at = index.cpu().numpy(), bits_of(c.k_pool), 0
    for r in range(R):
        page, row = c.place(r, c.total[r])
        x = got[page, :, row].astype(np.float64)
        s = slice(c.cu[r], c.cu[r + 1])
        ref = po.key_weights(f64(q[s]), lse[s], f64(c.k_rows[r]), starts[r], d ** -0.5, 1.0, None) if lens[r] else np.zeros((starts[r], H_kv))
        assert (np.abs(x - ref) <= rtol * ref).all(), r
        to_page, to_row = c.place(r, kept[r], new_table[r])
        for g in range(H_kv):
            want = po.rows_kept(x[:, g], kept[r], first[r], recent[r])
            assert np.array_equal(idx[at:at + kept[r]], want), (r, g)
            assert np.array_equal(k_got[to_page, g, to_row], c.k_rows[r][want, g])
            at += kept[r]


@pytest.mark.gpu
def test_a_captured_call_of_few_pages_replays_and_one_of_many_is_refused():
    import torch
    c = Paged(81, 8, 2, 128, 32, [1, 1, 6], [700, 31, 95]).fill()
    sh = AT.make_attn_shape(8, 2, 128, "f32")
    q, ws = c.dev(c.bf16(c.T, 8, 128)), c.workspace()
    o, z = torch.zeros(c.T, 8, 128, device="cuda"), torch.zeros(c.T, 8, device="cuda")
    w = torch.zeros(c.k_np.shape[0], 2, 32, device="cuda")

    def step():
        PG.attn_paged_prefill(sh, q, None, c.cu, c.starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids, o, z, ws)
        PG.attn_key_weights(sh, q, z, c.cu, c.starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w, ws)

    big = Paged(82, 4, 2, 64, 16, [1] * 4, [9000] * 4).fill()
    assert big.page_ids.size > 1792
    qb, big_ws = big.dev(big.bf16(big.T, 4, 64)), big.workspace()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
        for _ in range(10):                                                   # more than there are buffers
            with pytest.raises(B.GdnError) as e:
                PG.attn_paged_prefill(big.shape, qb, None, big.cu, big.starts, big.k_pool, big.v_pool, big.page_cu, big.page_ids, qb, None, big_ws)
            assert e.value.code < -1000                                        # the capture's own error
    torch.cuda.synchronize()
    for i in range(4):
        q.copy_(c.dev(c.bf16(c.T, 8, 128)))
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (o, z, w)]
        for x in (o, z, w):
            x.fill_(float("nan"))
        if i == 2:                                                            # other work of the same kind between two replays
            ob, zb = run_attend(big, big.bf16(big.T, 4, 64), None, "f32")
            assert bool(torch.isfinite(ob).all()) and bool(torch.isfinite(zb).all())
        g.replay()
        torch.cuda.synchronize()
        for r in range(3):
            page, row = c.place(r, c.total[r])
            page, row = torch.from_numpy(page.astype(np.int64)).cuda(), torch.from_numpy(row).cuda()
            assert torch.equal(w[page, :, row], want[2][page, :, row])
        assert torch.equal(o, want[0]) and torch.equal(z, want[1])


@pytest.mark.gpu
def test_one_token_given_by_heads_first():
    """A token whose heads were the first dimension of a tensor of one token: its token stride says nothing."""
    import torch
    c = Paged(83, 8, 2, 64, 16, [1], [40]).fill()
    rope, ws = PG.make_attn_rope(PG.attn_rope_freqs(64)[0]), c.workspace()
    x = [c.dev(c.bf16(1, h, 64)) for h in (8, 2, 2)]
    got = []
    for turn in (False, True):
        k, v, out = c.k_pool.clone(), c.v_pool.clone(), torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda")
        q_, k_, v_ = [t.reshape(-1, 1, 64).clone().transpose(0, 1) if turn else t for t in x]
        PG.attn_rope_append(c.shape, rope, q_, k_, v_, c.cu, None, c.starts, k, v, c.page_cu, c.page_ids, out, ws)
        got.append((bits_of(out), bits_of(k), v.cpu().numpy().view(np.int16)))
    for a, b in zip(*got):
        assert np.array_equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts", [
    (16, 2, 128, 64, [1], [900]), (6, 2, 64, 16, [1, 0, 1, 1], [975, 12, 512, 640]), (4, 2, 256, 32, [1, 5], [300, 470]),
    (8, 8, 128, 256, [14, 13], [668, 705]), (8, 1, 256, 16, [30], [1700]), (32, 4, 64, 32, [3, 1], [767, 1100]),   # (the last beside a few-rows request)
    (2, 1, 128, 16, [1, 200], [5000, 600]), (1, 1, 256, 128, [300], [0]),
])
def test_short_walks_cut_in_small_calls(H_q, H_kv, d, P, lens, starts):
    """Cut or whole, the same values; where a later token's rows are not numbers, the earlier ones' are."""
    import torch
    c = Paged(91, H_q, H_kv, d, P, lens, starts, stride_pad=8).fill()
    q, g = c.bf16(c.T, H_q, d, s=2.0), c.bf16(c.T, H_q, d)
    o, z = run_attend(c, q, g, "f32")
    check_attend(c, q, g, "f32", o, z)
    r = int(np.argmax(lens))
    page, row = c.place(r, c.total[r])
    c.view(c.v_np)[page[-1], :, row[-1]] = np.inf                            # what the longest request's last token brings
    c.view(c.k_np)[page[-1], :, row[-1]] = 0x7fc0
    c.fill_values()
    o2, z2 = run_attend(c, q, g, "f32")
    last = int(c.cu[r + 1]) - 1
    assert bool(torch.isnan(o2[last]).all()) and bool(torch.isnan(z2[last]).all())
    o2[last], z2[last] = o[last], z[last]
    check_attend(c, q, g, "f32", o2, z2)


# ----------------------------------------------------------------------------- what else is refused
@pytest.mark.parametrize("over", [
    dict(q=FakePool(0x10000, (9, 4, 64), 512), q_out=FakePool(0x10000, (9, 4, 64))),          # in place, but the queries lie apart
    dict(rope=PG.make_attn_rope(np.ones(32), in_dtype="f32"), q_out=FakePool(0x10000, (9, 4, 64))),   # ... or are twice as wide
    dict(q_out=FakePool(0x10010, (9, 4, 64))),                                                # ... or begin elsewhere
    dict(q_out=FakePool(0x10000 + 4608 - 16, (9, 4, 64))),                                    # over the last query
    dict(q_out=FakePool(0x20000 - 4608 + 16, (9, 4, 64))), dict(q_out=FakePool(0x20000 + 2304 - 16, (9, 4, 64))),   # over the first and the last key
    dict(v=FakePool(0x30000, (9, 2, 64), 1024), q_out=FakePool(0x30000 + 8 * 2048, (9, 4, 64))),                    # over a value
])
def test_rope_append_refuses_an_output_over_its_inputs(no_stream, over):
    """q_out over q that is not q itself, packed and bf16, or over k or v: workgroups would write what others have yet to read."""
    a = dict(CALL, rope=PG.make_attn_rope(np.ones(32)), q=X, k=FakePool(0x20000, (9, 2, 64)), v=FakePool(0x30000, (9, 2, 64)), pos=[0, 100],
             q_out=FakePool(0x40000, (9, 4, 64)))
    a.update(over)
    refused(PG.attn_rope_append, -7, a["shape"], a["rope"], a["q"], a["k"], a["v"], a["cu_seqlens"], a["pos"], a["start"], a["k_pool"], a["v_pool"],
            a["page_cu"], a["page_ids"], a["q_out"], a["workspace"])


def test_rope_append_refuses_too_many_heads_before_anything_is_enqueued(no_stream):
    """More pieces to a token than its kernel numbers, in a call whose plan is long enough for a launch of its own."""
    n, heads = 200, 1 << 26
    q = FakePool(0x1000000, (n, heads, 64), nbytes=1 << 50)
    kv = FakePool(0x10000, (n, 1, 64))
    pool = FakePool(0x200000, (n, 1, 16, 64))
    refused(PG.attn_rope_append, -3, AT.make_attn_shape(heads, 1, 64), PG.make_attn_rope(np.ones(32)), q, kv, kv, np.arange(n + 1), None, np.zeros(n, np.int32),
            pool, pool, np.arange(n + 1), np.arange(n), FakePool(1 << 50, (n, heads, 64), nbytes=1 << 50), FakePool(0x100000, nbytes=1 << 45))


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts", [
    (4, 2, 128, 16, [40], [300]), (8, 1, 64, 32, [5, 70], [500, 10]), (6, 2, 256, 64, [9, 21], [20, 700]), (16, 2, 128, 64, [1100], [40]),   # (cut rows)
    (16, 2, 128, 16, [1, 2], [90, 33]),                                       # the few-rows kernel
])
def test_key_weights_of_a_key_that_every_row_gives_minus_infinity(H_q, H_kv, d, P, lens, starts):
    """An element of a cached key is -infinity and positive in every query: its weight is 0, also beside rows that fill a tile's end."""
    import torch
    c = Paged(63, H_q, H_kv, d, P, lens, starts)
    at = [s // 2 for s in starts]
    for k, j in zip(c.k_rows, at):
        k[j, :, 5] = 0xff80
    c.fill()
    q = c.bf16(c.T, H_q, d)
    q[..., 5] = 0x3f80                                 # 1
    lse = np.zeros((c.T, H_q), np.float32)
    finite = [k.copy() for k in c.k_rows]
    for r in range(len(lens)):
        s = slice(c.cu[r], c.cu[r + 1])
        lse[s] = po.row_lse(f64(q[s]), f64(c.k_rows[r]), starts[r], d ** -0.5)
        finite[r][at[r], :, 5] = 0
    assert np.isfinite(lse).all()
    w = torch.full((c.k_np.shape[0], H_kv, P), float("nan"), device="cuda")
    PG.attn_key_weights(c.shape, c.dev(q), torch.from_numpy(lse).cuda(), c.cu, starts, c.k_pool, c.page_cu, c.page_ids, 1.0, None, w, c.workspace())
    w = w.cpu().numpy().astype(np.float64)
    held, c.k_rows = c.k_rows, finite
    rtol = np.expm1(logit_error(c, q) + 2.0 ** -22 * (1 + np.abs(lse).max())) + (max(lens) * (H_q // H_kv) + 8) * 2.0 ** -24
    for r in range(len(lens)):
        s = slice(c.cu[r], c.cu[r + 1])
        page, row = c.place(r, c.total[r])
        ref = po.key_weights(f64(q[s]), lse[s], f64(held[r]), starts[r], d ** -0.5, 1.0, None)
        assert (ref[at[r]] == 0).all() and (np.abs(w[page, :, row] - ref) <= rtol * ref).all(), r


@pytest.mark.gpu
def test_a_stream_that_stands_still_holds_up_no_call_on_another():
    """More calls with long page tables behind half a second of other work than there are staging buffers, and one on another stream: each returns in
    milliseconds, and all come out right."""
    import time
    import torch
    c = Paged(72, 4, 2, 64, 16, [1] * 20, [1500 + 20 * i for i in range(20)]).fill()
    assert c.page_ids.size > 1792
    q = c.bf16(c.T, 4, 64)
    want, wz = run_attend(c, q, None, "f32")
    qd, sh = c.dev(q), AT.make_attn_shape(4, 2, 64, "f32")
    outs = [(torch.zeros(c.T, 4, 64, device="cuda"), torch.zeros(c.T, 4, device="cuda"), c.workspace()) for _ in range(13)]

    def call(i, stream=None):
        o, z, ws = outs[i]
        PG.attn_paged_prefill(sh, qd, None, c.cu, c.starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids, o, z, ws, stream)

    for i in range(13):                     # every buffer there is has been made
        call(i)
    for o, z, _ in outs:
        o.fill_(float("nan"))
        z.fill_(float("nan"))
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda._sleep(1 << 20)
    a.record()
    torch.cuda._sleep(1 << 22)
    b.record()
    torch.cuda.synchronize()
    cycles = int((1 << 22) * 500 / a.elapsed_time(b))                          # of half a second
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(cycles)
    t0 = time.perf_counter()
    for i in range(12):
        call(i, side)
    call(12)
    host = time.perf_counter() - t0
    torch.cuda.synchronize()
    for o, z, _ in outs:
        assert torch.equal(o, want) and torch.equal(z, wz)
    assert host < 0.2, host


@pytest.mark.gpu
def test_threads_with_streams_of_their_own_keep_their_own_plans():
    import threading
    import torch
    c = Paged(73, 4, 2, 64, 16, [1] * 24, [1200 + 30 * i for i in range(24)]).fill()
    assert c.page_ids.size > 1792
    q = c.bf16(c.T, 4, 64)
    want, wz = run_attend(c, q, None, "f32")
    torch.cuda.synchronize()
    qd, sh = c.dev(q), AT.make_attn_shape(4, 2, 64, "f32")
    work = []
    for t in range(4):
        rng, stream, ws = np.random.default_rng(t), torch.cuda.Stream(), c.workspace()
        stream.wait_stream(torch.cuda.current_stream())
        calls = []
        for i in range(20):
            order = rng.permutation(24)
            at = torch.from_numpy(order).cuda()
            tables = [c.table[r] for r in order]
            calls.append((at, qd[at].contiguous(), np.asarray(c.starts)[order], np.concatenate([[0], np.cumsum([x.size for x in tables])]), np.concatenate(tables),
                          torch.zeros(24, 4, 64, device="cuda"), torch.zeros(24, 4, device="cuda")))
        work.append((stream, ws, calls))
    torch.cuda.synchronize()
    failed = []

    def run(stream, ws, calls):
        try:
            for at, qt, st, tcu, ids, o, z in calls:
                PG.attn_paged_prefill(sh, qt, None, np.arange(25), st, c.k_pool, c.v_pool, tcu, ids, o, z, ws, stream)
        except Exception as e:              # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for _, _, calls in work:
        for at, _, _, _, _, o, z in calls:
            assert torch.equal(o, want[at]) and torch.equal(z, wz[at])


def attend_with_not_finite_values(q, k, v, start, scale):
    """The definition row by row: what a row does not see adds nothing, a weight above 0 times an infinity is that infinity."""
    n, H_q, d = q.shape
    G = H_q // k.shape[1]
    finite = np.where(np.isfinite(v), v, 0.0)
    o = ao.attention_suffix(q, k, finite, start, scale)
    plus, minus, nan = (np.cumsum(x, 0) > 0 for x in (v == np.inf, v == -np.inf, np.isnan(v)))
    for t in range(n):
        for x, what in ((plus, np.inf), (minus, -np.inf), (nan, np.nan)):
            with np.errstate(invalid="ignore"):         # (infinities of both signs)
                o[t] += np.where(np.repeat(x[start + t], G, 0), what, 0.0)
    return o


NOT_FINITE = [  # H_q, H_kv, d, P, lens, starts
    (4, 2, 64, 16, [40], [3]), (16, 2, 128, 32, [24, 5], [100, 60]), (6, 2, 64, 64, [200], [63]), (8, 8, 256, 64, [70], [400]), (32, 4, 128, 128, [400], [600]),
    (1, 1, 128, 16, [129], [0]), (2, 2, 256, 16, [300], [17]),
    (4, 1, 128, 16, [3], [1300]), (1, 1, 64, 32, [9], [1100]), (8, 8, 256, 64, [14], [1500]), (16, 2, 64, 128, [2, 2, 2], [1024, 1500, 3000]),   # few rows
]


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts", NOT_FINITE)
@pytest.mark.parametrize("kind", ["cached", "column", "column of the new", "signs"])
def test_values_that_are_not_finite_reach_the_rows_and_columns_that_see_them(H_q, H_kv, d, P, lens, starts, kind):
    """cached: one such value in front of the chunk.  column: a column of infinities, seen and unseen.  signs: infinities of both signs and a NaN among the new
    rows, in three columns of which one has all of them.  Everything else stays finite and right."""
    import torch
    c = Paged(64, H_q, H_kv, d, P, lens, starts)
    for r, (n, s) in enumerate(zip(lens, starts)):
        v = c.v_rows[r]
        if kind == "cached":
            v[s // 2, 0, 7] = np.inf
            v[(s + n) // 2, -1, 9] = np.nan
        elif kind == "column":
            v[:, 0, 33] = np.inf
        elif kind == "column of the new":
            v[s:, 0, 33] = -np.inf
        else:
            at = s + np.arange(n)
            v[at[n // 3], :, 1] = np.inf
            v[at[n // 2], :, 1] = -np.inf
            v[at[n // 3], :, 40] = -np.inf
            v[at[-1], :, 1] = v[at[-1], :, 63] = np.nan
    c.fill()
    q = c.bf16(c.T, H_q, d, s=0.5)                     # (no weight rounds to 0)
    o, z = run_attend(c, q, None, "f32")
    o, z = o.double().cpu().numpy(), z.double().cpu().numpy()
    le = logit_error(c, q)
    for r in range(len(lens)):
        s = slice(c.cu[r], c.cu[r + 1])
        k, v = f64(c.k_rows[r]), c.v_rows[r].astype(np.float64)
        ref = attend_with_not_finite_values(f64(q[s]), k, v, starts[r], d ** -0.5)
        ok = np.isfinite(ref)
        assert ((o[s] == ref) | (np.isnan(o[s]) & np.isnan(ref)))[~ok].all(), (r, np.argwhere(~ok & (o[s] != ref) & ~np.isnan(ref))[:5])
        assert (np.abs(o[s] - np.where(ok, ref, 0.0))[ok] <= 2.0 ** -8 * np.abs(v[np.isfinite(v)]).max()).all(), r
        zr = po.row_lse(f64(q[s]), k, starts[r], d ** -0.5)
        assert (np.abs(z[s] - zr) <= le + 2.0 ** -20 * (1 + np.abs(zr))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,lens,starts", [(16, 2, 128, [400], [6000]), (8, 2, 64, [600, 300], [3000, 2500]), (8, 8, 128, [8] * 32, [4000] * 32)])
@pytest.mark.parametrize("kind", ["cached", "column"])
def test_values_that_are_not_finite_cost_no_more_than_a_few_walks(H_q, H_kv, d, lens, starts, kind):
    """One bad value among the cached rows, or an overflown column of all rows: a call may walk again what it has to, at the speed of a walk."""
    import torch
    c = Paged(65, H_q, H_kv, d, 64, lens, starts).fill()
    q = c.dev(c.bf16(c.T, H_q, d, s=0.5))
    sh = AT.make_attn_shape(H_q, H_kv, d, "bf16")
    o, ws = torch.zeros(c.T, H_q, d, dtype=torch.bfloat16, device="cuda"), c.workspace()

    def best():
        times = []
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            PG.attn_paged_prefill(sh, q, None, c.cu, c.starts, c.k_pool, c.v_pool, c.page_cu, c.page_ids, o, None, ws)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    clean = best()
    for r in range(len(lens)):
        page, row = c.place(r, c.total[r])
        if kind == "cached":
            c.v_pool[int(page[5]), :, int(row[5]), 3] = float("nan")
        else:
            c.v_pool[torch.from_numpy(page.astype(np.int64)).cuda(), :, torch.from_numpy(row).cuda(), 3] = float("inf")
    bad = best()
    assert not bool(torch.isfinite(o[:, :, 3].float()).any()) and bool(torch.isfinite(o[:, :, :3].float()).all())
    assert bad <= (1.5 if kind == "cached" else 40) * clean, (clean, bad)


@pytest.mark.parametrize("over", [dict(cu_seqlens=[0, 5]), dict(cu_seqlens=[0, 5, 9, 9]), dict(page_cu=[0, 1]), dict(page_cu=[0, 1, 3, 3]), dict(page_ids=[7, 3]),
                                  dict(page_ids=[])])
def test_index_arrays_shorter_than_the_call_reads_are_refused(no_stream, over):
    a = dict(CALL, **over)
    arrays = a["k_pool"], a["page_cu"], a["page_ids"]
    rope, kv, lse = PG.make_attn_rope(np.ones(32)), FakePool(0x20000, (9, 2, 64)), FakePool(0x30000)
    for pos in (None, [0, 100], [0], [0, 1, 2]):
        with pytest.raises(ValueError):
            PG.attn_rope_append(a["shape"], rope, X, kv, kv, a["cu_seqlens"], pos, a["start"], a["k_pool"], *arrays, X, WS)
    with pytest.raises(ValueError):
        PG.attn_rope_append(CALL["shape"], rope, X, kv, kv, CALL["cu_seqlens"], [0], CALL["start"], K_POOL, V_POOL, CALL["page_cu"], CALL["page_ids"], X, WS)
    with pytest.raises(ValueError):
        PG.attn_paged_prefill(a["shape"], X, None, a["cu_seqlens"], a["start"], a["k_pool"], *arrays, X, None, WS)
    with pytest.raises(ValueError):
        PG.attn_key_weights(a["shape"], X, lse, a["cu_seqlens"], a["start"], *arrays, 1.0, None, W_POOL, WS)
    evict = dict(rows=[5, 24], keep=[4, 10], first=[2, 2], recent=[2, 3], page_cu=[0, 1, 3], page_ids=[7, 3, 39], new_page_cu=[0, 1, 2], new_page_ids=[1, 2])
    for over in (dict(rows=[5]), dict(keep=[4]), dict(first=[2, 2, 2]), dict(recent=[]), dict(page_cu=[0, 1]), dict(page_ids=[7, 3]), dict(new_page_cu=[0, 1]),
                 dict(new_page_ids=[1])):
        e = dict(evict, **over)
        with pytest.raises(ValueError):
            PG.attn_evict(CALL["shape"], e["rows"], e["keep"], e["first"], e["recent"], K_POOL, V_POOL, W_POOL, e["page_cu"], e["page_ids"], e["new_page_cu"],
                          e["new_page_ids"], FakePool(), WS)


def test_tensors_of_another_type_than_the_kernels_read_are_refused(no_stream):
    import torch
    bf16, f16, f32, i32 = torch.bfloat16, torch.float16, torch.float32, torch.int32
    cu, st, tcu, ids = [0, 5, 9], [0, 20], [0, 1, 3], [7, 3, 39]
    ws = FakePool(0x100000, nbytes=64)
    pool, w, x, kv, z, i = (torch.zeros(*n) for n in ((40, 2, 16, 64), (40, 2, 16), (9, 4, 64), (9, 2, 64), (9, 4), (99,)))

    def append(in_dtype, q, k, v, kp, vp, out):
        PG.attn_rope_append(AT.make_attn_shape(4, 2, 64), PG.make_attn_rope(np.ones(32), in_dtype=in_dtype), x.to(q), kv.to(k), kv.to(v), cu, None, st, pool.to(kp),
                            pool.to(vp), tcu, ids, x.to(out), ws)

    def attend(o_dtype, q, gate, kp, vp, o, lse):
        PG.attn_paged_prefill(AT.make_attn_shape(4, 2, 64, o_dtype), x.to(q), x.to(gate), cu, st, pool.to(kp), pool.to(vp), tcu, ids, x.to(o), z.to(lse), ws)

    def weigh(q, lse, kp, wi, wo):
        PG.attn_key_weights(AT.make_attn_shape(4, 2, 64), x.to(q), z.to(lse), cu, st, pool.to(kp), tcu, ids, 1.0, w.to(wi), w.to(wo), ws)

    def evict(kp, vp, wp, index):
        PG.attn_evict(AT.make_attn_shape(4, 2, 64), [5, 24], [4, 9], [1, 1], [1, 1], pool.to(kp), pool.to(vp), w.to(wp), tcu, ids, [0, 1, 2], [1, 2], i.to(index), ws)

    for call, right in ((append, ("bf16", bf16, bf16, bf16, bf16, f16, bf16)), (append, ("f32", f32, f32, f32, bf16, f16, bf16)),
                        (attend, ("bf16", bf16, bf16, bf16, f16, bf16, f32)), (attend, ("f32", bf16, bf16, bf16, f16, f32, f32)),
                        (weigh, (bf16, f32, bf16, f32, f32)), (evict, (bf16, f16, f32, i32))):
        ws._n = 64
        refused(call, -9, *right)                                             # nothing else is wrong: the workspace is too small
        ws._n = 1 << 30
        for at, want in enumerate(right):
            for other in (bf16, f16, f32, i32, torch.int16, torch.float64):
                if not isinstance(want, str) and other is not want:
                    refused(call, -3, *right[:at], other, *right[at + 1:])


@pytest.mark.parametrize("x", [[3, 1, 2], (3, 1, 2), np.array([3, 1, 2]), np.array([3, 9, 1, 9, 2, 9], np.int32)[::2], np.arange(4, 0, -1, dtype=np.int32)[1:][[0, 2, 1]]])
def test_index_arrays_of_any_kind_arrive_as_they_are(x):
    read_only = np.array(x, np.int32)
    read_only.flags.writeable = False
    for a in (x, read_only):
        got = PG._array(3, a)
        assert list((ctypes.c_int32 * 3).from_address(ctypes.addressof(got))) == [3, 1, 2]


def test_tensors_shorter_than_the_call_are_refused(no_stream):
    """Of each of a call's tensors one element or row less than it reads or writes."""
    import torch
    bf16 = torch.bfloat16
    cu, st, tcu, ids = [0, 5, 9], [0, 20], [0, 1, 3], [7, 3, 39]
    ws = FakePool(0x100000, nbytes=64)
    k, v, w = torch.zeros(40, 2, 16, 64, dtype=bf16), torch.zeros(40, 2, 16, 64, dtype=torch.float16), torch.zeros(40, 2, 16)
    x, kv, z, i = torch.zeros(9, 4, 64, dtype=bf16), torch.zeros(9, 2, 64, dtype=bf16), torch.zeros(9, 4), torch.zeros(26, dtype=torch.int32)
    sh, rope = AT.make_attn_shape(4, 2, 64, "bf16"), PG.make_attn_rope(np.ones(32))
    calls = [(lambda q, k_, v_, out: PG.attn_rope_append(sh, rope, q, k_, v_, cu, None, st, k, v, tcu, ids, out, ws), (x, kv, kv, x)),
             (lambda q, gate, o, lse: PG.attn_paged_prefill(sh, q, gate, cu, st, k, v, tcu, ids, o, lse, ws), (x, x, x, z)),
             (lambda q, lse: PG.attn_key_weights(sh, q, lse, cu, st, k, tcu, ids, 1.0, w, w, ws), (x, z)),
             (lambda index: PG.attn_evict(sh, [5, 24], [4, 9], [1, 1], [1, 1], k, v, w, tcu, ids, [0, 1, 2], [1, 2], index, ws), (i,))]
    for call, right in calls:
        ws._n = 64
        refused(call, -9, *right)                                             # nothing else is wrong: the workspace is too small
        ws._n = 1 << 30
        for at, t in enumerate(right):
            refused(call, -3, *right[:at], t[:-1], *right[at + 1:])
    refused(calls[3][0], -3, torch.zeros(0, dtype=torch.int32))
    refused(lambda: PG.attn_evict(sh, [5, 24], [4, 90], [1, 1], [1, 1], k, v, w, tcu, ids, [0, 1, 3], [1, 2, 4], torch.zeros(55, dtype=torch.int32), ws), -3)


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,lens,starts", [
    (16, 2, 128, 64, [1, 1, 1], [3000, 1023, 1500]), (4, 4, 64, 16, [1], [9000]), (8, 1, 256, 128, [2, 1], [1100, 2047]), (32, 4, 64, 32, [2] * 9, [1024 + 211 * i for i in range(9)]),
    (16, 2, 128, 64, [1] * 40, [1100 + 150 * i for i in range(40)]),          # few-rows walks, cut
    (8, 8, 64, 64, [1] * 66, [1024 + 3 * i for i in range(66)]),              # ... and whole
    (16, 2, 128, 64, [600] * 8, [500 + 30 * i for i in range(8)]),            # the 128-row kernel's in a call that fills the chip
    (16, 4, 64, 32, [500, 700, 640, 1] * 4, [40, 900, 0, 1300] * 4),
])
def test_walks_that_both_forms_plan_alike_have_the_same_bits(H_q, H_kv, d, P, lens, starts):
    """Walks cut and whole as the planner likes: requests of few rows behind 1024 and more, and calls that are not cut.  Where a walk has more than 16 parts the
    forms merge them in different orders: the same values."""
    import torch
    R = len(lens)
    c = Paged(210, H_q, H_kv, d, P, lens, starts)
    v_new = [wl.f32_to_bf16_bits(v[s:].astype(np.float32)) for v, s in zip(c.v_rows, starts)]
    cap = max(c.total)
    kc, vc = np.zeros((R, cap, H_kv, d), np.uint16), np.zeros((R, cap, H_kv, d), np.float16)
    for r in range(R):
        c.v_rows[r][starts[r]:] = wl.to_f32(v_new[r]).astype(np.float16)
        kc[r, :starts[r]], vc[r, :starts[r]] = c.k_rows[r][:starts[r]], c.v_rows[r][:starts[r]]
    c.fill()
    q = c.bf16(c.T, H_q, d)
    o, _ = run_attend(c, q, None, "f32", lse=False)
    sh = AT.make_attn_shape(H_q, H_kv, d, "f32")
    os_ = torch.zeros_like(o)
    ws = torch.empty(AT.attn_workspace_bytes(sh, R, c.T), dtype=torch.uint8, device="cuda")
    AT.attn_suffix_prefill(sh, c.dev(q), c.dev(np.concatenate([k[s:] for k, s in zip(c.k_rows, starts)])), c.dev(np.concatenate(v_new)), None, c.cu, starts,
                           c.dev(kc), torch.from_numpy(vc).cuda(), list(range(R)), os_, ws)
    units, _, _ = AT.attn_plan(sh, c.cu, starts)
    if np.unique(units[:, :2], axis=0, return_counts=True)[1].max() <= 16:
        assert torch.equal(o, os_)
    else:
        check_attend(c, q, None, "f32", o, None)
        check_attend(c, q, None, "f32", os_, None)


@pytest.mark.gpu
@pytest.mark.parametrize("H_q,H_kv,d,P,R,n,lo,hi,whole", [
    (16, 8, 64, 64, 100, 1, 1024, 1300, True), (16, 8, 64, 32, 70, 2, 1023, 1200, True), (8, 8, 128, 16, 96, 1, 1030, 1400, True),
    (16, 2, 256, 128, 260, 1, 1024, 1100, True), (16, 8, 256, 64, 66, 4, 1030, 1100, True), (32, 4, 128, 64, 130, 2, 1024, 1300, True),
    (16, 2, 128, 64, 16, 1, 9000, 10000, False),                              # as many bytes, walks cut
])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_batches_of_few_rows_whose_walks_stay_whole(H_q, H_kv, d, P, R, n, lo, hi, whole, dtype):
    """More requests and heads than workgroups to cut them into, and more bytes than the last cache keeps, gated and with log-sum-exps.  Where a request has
    several tokens, the last brings an infinity and a NaN, which the rows before it do not see."""
    import torch
    gen, rng = torch.Generator(device="cuda").manual_seed(3), np.random.default_rng(4)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    starts = rng.integers(lo, hi, R)
    pages = -(-(starts + n) // P)
    tcu = np.concatenate([[0], np.cumsum(pages)])
    ids = rng.permutation(int(tcu[-1])).astype(np.int32)
    k, v = normal(ids.size, H_kv, P, d).bfloat16(), normal(ids.size, H_kv, P, d).half()
    q, gate = normal(R * n, H_q, d).bfloat16(), normal(R * n, H_q, d).bfloat16()
    cu = np.arange(R + 1) * n
    places = []
    for r in range(R):
        j = np.arange(starts[r] + n)
        places.append((torch.from_numpy(ids[tcu[r] + j // P].astype(np.int64)).cuda(), torch.from_numpy(j % P).cuda()))
        if n > 1:
            v[places[r][0][-1], :, places[r][1][-1], 5] = float("inf")
            v[places[r][0][-1], :, places[r][1][-1], d - 1] = float("nan")
    sh = AT.make_attn_shape(H_q, H_kv, d, dtype)
    units, _, _ = AT.attn_plan(sh, cu, starts)
    assert (units[:, 4] == -1).all() == whole and int((starts + n).sum()) * H_kv * d * 4 > 1 << 27
    o, z = torch.full((R * n, H_q, d), float("nan"), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda"), torch.full((R * n, H_q), float("nan"), device="cuda")
    ws = torch.full((PG.attn_paged_workspace_bytes(sh, R, R * n, ids.size),), 0xA5, dtype=torch.uint8, device="cuda")
    PG.attn_paged_prefill(sh, q, gate, cu, starts, k, v, tcu, ids, o, z, ws)
    o2 = torch.zeros_like(o)
    PG.attn_paged_prefill(sh, q, gate, cu, starts, k, v, tcu, ids, o2, None, ws)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16))
    G, step = 2.0 ** -8, 2.0 ** -8 if dtype == "bf16" else 0.0
    for r in range(R):
        page, row = places[r]
        kr, vr = k[page, :, row].double(), v[page, :, row].double()           # [rows][H_kv][d]
        for t in range(n):
            seen = starts[r] + t + 1
            qt = q[r * n + t].double().view(H_kv, -1, d)
            x = torch.stack([qt[g] @ kr[:seen, g].T.contiguous() for g in range(H_kv)]) * d ** -0.5
            zr = torch.logsumexp(x, -1)
            p = (x - zr[..., None]).exp()
            ref = torch.stack([p[g] @ vr[:seen, g] for g in range(H_kv)]).view(H_q, d) * torch.sigmoid(gate[r * n + t].double())
            got, zt = o[r * n + t].double(), z[r * n + t].double()
            le = (d + 16) * 2.0 ** -24 * d ** -0.5 * float(kr[:seen].norm(dim=-1).max() * qt.norm(dim=-1).max())
            assert bool(((zt - zr.view(-1)).abs() <= le + 2.0 ** -20 * (1 + zr.view(-1).abs())).all()), (r, t)
            if t == n - 1 and n > 1:
                assert bool((got[:, 5] == float("inf")).all()) and bool(got[:, d - 1].isnan().all())
                got[:, [5, d - 1]] = ref[:, [5, d - 1]] = 0.0
            top = float(vr[:seen].nan_to_num(0.0, 0.0, 0.0).abs().max())
            assert bool(((got - ref).abs() <= G * top + step * ref.abs()).all()), (r, t, float((got - ref).abs().max()))


@pytest.mark.gpu
@pytest.mark.parametrize("H_kv,P,rows,keep,first,recent,kind", [
    (2, 16, [32768, 32769], [3000, 3000], [4, 0], [64, 64], "normal"), (1, 64, [40961, 100], [40000, 7], [0, 1], [0, 1], "ties"),
    (1, 256, [200003], [1000], [4], [100], "normal"), (2, 128, [70000], [33000], [33], [64], "equal"), (1, 32, [90001], [45000], [8], [8], "tail"),
    (1, 32, [90001], [89000], [40000], [33000], "ties"),
])
def test_evict_from_more_rows_than_registers_hold(H_kv, P, rows, keep, first, recent, kind):
    """Requests of more than 32768 rows, whose later ranks are read again."""
    import torch
    d = 64
    new_n = [-(-m // P) for m in keep]
    c = Paged(33, H_kv, H_kv, d, P, [0] * len(rows), rows, extra=sum(new_n)).fill()
    w_np = np.full(c.k_np.shape[:1] + (H_kv, P), np.nan, np.float32)
    w_rows = []
    for r, n in enumerate(rows):
        w = c.rng.standard_normal((n, H_kv)).astype(np.float32)
        if kind == "ties":
            w = np.round(2 * w)
        if kind == "equal":
            w[:] = -1.5
        if kind == "tail":                              # what is kept lies behind the rows held
            w[:50000] -= 100.0
            w[60000::3] = np.nan
        w_rows.append(w)
        page, row = c.place(r, n)
        w_np[page, :, row] = w
    spare = list(c.spare)
    new_table = [np.array([spare.pop() for _ in range(m)], np.int32) for m in new_n]
    w_pool = torch.from_numpy(w_np).cuda()
    index = torch.full((sum(keep) * H_kv,), -7, dtype=torch.int32, device="cuda")
    PG.attn_evict(c.shape, rows, keep, first, recent, c.k_pool, c.v_pool, w_pool, c.page_cu, c.page_ids, np.concatenate([[0], np.cumsum(new_n)]),
                  np.concatenate(new_table), index, c.workspace(0, c.page_ids.size + sum(new_n)))
    idx, k_got, v_got, w_got, at = index.cpu().numpy(), bits_of(c.k_pool), bits_of(c.v_pool), w_pool.cpu().numpy(), 0
    for r in range(len(rows)):
        page, row = c.place(r, keep[r], new_table[r])
        for g in range(H_kv):
            want = po.rows_kept(w_rows[r][:, g], keep[r], first[r], recent[r])
            assert np.array_equal(idx[at:at + keep[r]], want), (r, g)
            at += keep[r]
            assert np.array_equal(k_got[page, g, row], c.k_rows[r][want, g]) and np.array_equal(v_got[page, g, row], c.v_rows[r][want, g].view(np.uint16))
            assert np.array_equal(w_got[page, g, row].view(np.uint32), w_rows[r][want, g].view(np.uint32))
