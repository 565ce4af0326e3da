"""The residual stream's norms (include/gdn_block.h) against their oracle (the definition in fp64, with a bound of fp32's error).

CPU part: oracle pins, exports, refusals (every check returns before a pointer is used).  GPU part (marked gpu): element by element.
Tolerance: the oracle's bound for outputs in fp32; one rounding more, 2^-8 of the value (half a step), for outputs in bf16.
"""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import block_oracle as bo
from paper_2605_05219_amd import binding as B, block as BL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ----------------------------------------------------------------------------- the oracle
def test_oracle_hand_worked_rows():
    y, r = np.array([[3.0, -4.0, 0.0, 0.0]]), np.array([[1.0, 1.0, 1.0, 1.0]])
    (s, _), (x, _) = bo.block_norm(y, None, np.ones(4), None, r, np.array([1.0, 2.0, 1.0, 1.0]), np.array([0.0, 0.0, 5.0, 0.0]), "rms", "layer",
                                   eps_post=0.0, eps_pre=0.0, scale=2.5)
    assert np.allclose(s, [[4.0, -3.0, 1.0, 1.0]], rtol=1e-15)           # rms of y is 2.5
    # s: mean 3/4, squares left (3.25, 3.75, .25, .25)^2 = 24.75 / 4
    sig = np.sqrt(24.75 / 4)
    assert np.allclose(x, [[3.25 / sig, -7.5 / sig, 0.25 / sig + 5, 0.25 / sig]], rtol=1e-15)
    (s, _), none = bo.block_norm(y, np.array([[2.0]]), None, None, None, None, None, "none", "none", scale=0.5)
    assert none is None and np.array_equal(s, y)
    (s, _), _ = bo.block_norm(y, np.zeros((1, 4)), None, None, r, None, None, "none", "none", "sigmoid")
    assert np.array_equal(s, r + y / 2)


def test_oracle_moments_and_invariance():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((5, 64)) * 3 + 2
    n, _ = bo.normalise(v, 0 * v, "layer", np.ones(64), None, 0.0, 0.0)
    assert np.allclose(n.mean(1), 0, atol=1e-14) and np.allclose((n * n).mean(1), 1)
    assert np.allclose(bo.normalise(7 * v - 3, 0 * v, "layer", np.ones(64), None, 0.0, 0.0)[0], n)
    m, _ = bo.normalise(v, 0 * v, "rms", np.zeros(64), None, 1.0, 0.0)
    assert np.allclose((m * m).mean(1), 1) and np.allclose(m / v, (m / v)[:, :1])


# ----------------------------------------------------------------------------- refusals
def test_library_exports_every_symbol_the_block_header_declares():
    header = open(os.path.join(ROOT, "include", "gdn_block.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(gdn_block_\w+)\s*\(", header))
    assert declared == set(BL.EXPORTS)
    L = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert getattr(L, name) is not None


def raw(shape=None, **over):
    a = dict(y=0x100000, ldy=256, w_post=0x700000, b_post=0x701000, r=0x200000, ldr=256, w_pre=0x702000, b_pre=0, s=0x300000, lds=256,
             x=0x400000, ldx=256, T=100, gate=0x500000, ldg=256)
    a.update(over)
    return BL.gdn_block_norm_raw(shape if shape is not None else BL.make_block_shape(256, "rms", "rms", gate="element"), **a)


def shaped(**over):
    a = dict(D=256, post="rms", pre="rms", gate="element")
    a.update(over)
    return BL.make_block_shape(**a)


def altered(field, value):
    s = shaped()
    setattr(s, field, value)
    return s


@pytest.mark.parametrize("shape,over,code", [
    (None, dict(T=-1), -11), (None, dict(T=1 << 31), -11), (None, dict(ldy=1 << 41), -11),
    (altered("D", 0), {}, -3), (altered("D", 32776), {}, -3), (altered("D", 250), {}, -2),
    (altered("in_dtype", 2), {}, -3), (altered("s_dtype", -1), {}, -3), (altered("x_dtype", 7), {}, -3),
    (altered("post", 3), {}, -3), (altered("pre", -1), {}, -3), (altered("gate", 4), {}, -3), (altered("gate_act", 2), {}, -3),
    (altered("eps_post", -1.0), {}, -3), (altered("eps_pre", float("nan")), {}, -3), (altered("eps_pre", float("inf")), {}, -3),
    (None, dict(y=0), -3),                                        # a post norm of nothing
    (shaped(post="none", gate="none"), dict(y=0, r=0), -1),
    (None, dict(w_post=0), -1), (None, dict(w_pre=0), -1), (None, dict(gate=0), -1), (None, dict(x=0), -1),
    (shaped(pre="none"), {}, -3), (shaped(pre="none"), dict(x=0, s=0), -1),
    (None, dict(ldy=248), -3), (None, dict(ldr=0), -3), (None, dict(lds=-256), -3), (None, dict(ldx=255), -3), (None, dict(ldg=128), -3),
    (None, dict(ldy=260), -2), (None, dict(ldg=257), -2), (None, dict(y=0x100008), -2), (None, dict(x=0x400002), -2), (None, dict(gate=0x500004), -2),
    (None, dict(w_post=0x700004), -2), (None, dict(b_post=0x701008), -2), (None, dict(w_pre=0x702002), -2),
    (shaped(gate="token"), dict(ldg=0), -3), (shaped(gate="token"), dict(gate=0x500001), -2), (shaped(gate="channel"), dict(gate=0x500008), -2),
    (None, dict(s=0x400000), -7),                                 # one place for both outputs
    (None, dict(s=0x100010, lds=256), -7),                        # eight elements behind the input's rows
    (None, dict(x=0x200000, ldx=264), -7),                        # the same address, another stride
    (shaped(s_dtype="f32"), dict(s=0x100000), -7),                # the same rows, another type
    (None, dict(x=0x700000 - 256), -7),                           # over the weights
    (shaped(gate="token"), dict(ldg=1, s=0x500000), -7), (shaped(gate="channel"), dict(x=0x500000), -7),
])
def test_refusals(shape, over, code):
    assert raw(shape, **over) == code


def test_no_tokens_is_legal_and_touches_nothing():
    assert raw(T=0, y=0, r=0, s=0, x=0, gate=0) == 0


def overlap(a, b):
    """Whether rows (address, rows, pitch, width in bytes) share a byte, by listing them."""
    spans = [[(p + i * pitch, p + i * pitch + w) for i in range(n)] for p, n, pitch, w in (a, b)]
    return any(lo < y and x < hi for lo, hi in spans[0] for x, y in spans[1])


def test_columns_of_a_wider_buffer_are_told_from_rows_that_overlap():
    """Outputs beside, inside and across the rows of an input: refused where a byte is shared, let through where not.  T = 1 and the
    pairs of strides that differ may be refused without need, never let through wrongly."""
    shape = BL.make_block_shape(64, "none", "none")
    rng, let = np.random.default_rng(3), 0
    # (what is let through would be launched: without a device, or with the null stream's error, it ends in an error of another kind)
    import torch
    if torch.cuda.is_available():
        pytest.skip("calls that are let through would run")
    for _ in range(3000):
        T = int(rng.integers(1, 6))
        ldy, lds = 8 * int(rng.integers(8, 30)), 8 * int(rng.integers(8, 30))
        if rng.random() < 0.6:
            lds = ldy
        y = 0x100000
        s = y + 16 * int(rng.integers(-60, 200))
        code = BL.gdn_block_norm_raw(shape, y=y, ldy=ldy, s=s, lds=lds, T=T)
        shares, same = overlap((y, T, 2 * ldy, 128), (s, T, 2 * lds, 128)), s == y and (lds == ldy or T == 1)
        if shares and not same:
            assert code == -7
        elif ldy == lds or T == 1:
            assert code <= -1000 or code == 0
            let += 1
    assert let > 300


def test_python_binding_refuses_mismatched_tensors():
    import torch
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16)  # noqa: E731
    shape, w = BL.make_block_shape(64, "rms", "rms"), torch.zeros(64)
    good = dict(y=bf(4, 64), gate=None, w_post=w, b_post=None, r=bf(4, 64), w_pre=w, b_pre=None, s=bf(4, 64), x=bf(4, 64))
    for over in (dict(y=None, r=None), dict(y=bf(4, 72)), dict(r=bf(5, 64)), dict(s=torch.zeros(4, 64)), dict(x=bf(4, 128)[:, ::2]), dict(w_post=torch.zeros(63)),
                 dict(w_pre=torch.zeros(64, dtype=torch.float64)), dict(b_pre=torch.zeros(128)[::2]), dict(y=bf(256))):
        with pytest.raises(ValueError):
            BL.gdn_block_norm(shape, **{**good, **over})
    token = BL.make_block_shape(64, "rms", "rms", gate="token")
    for gate in (bf(4, 1), bf(5), torch.zeros(4)):
        with pytest.raises(ValueError):
            BL.gdn_block_norm(token, **{**good, "gate": gate})
    with pytest.raises(B.GdnError) as ei:                        # row strides that are no multiple of 8
        BL.gdn_block_norm(shape, **{**good, "x": bf(4, 68)[:, :64]})
    assert ei.value.code == -2
    with pytest.raises(B.GdnError) as ei:
        BL.gdn_block_norm(shape, **{**good, "r": bf(64).expand(4, 64)})
    assert ei.value.code == -3


# ----------------------------------------------------------------------------- GPU
DT = {}


def dt(name):
    import torch
    DT.update(bf16=torch.bfloat16, f32=torch.float32)
    return DT[name]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Call:
    def __init__(self, T, D, post="none", pre="rms", dtype="bf16", s_dtype="bf16", x_dtype="bf16", gate="none", gate_act="none", scale=1.0, offset=0.0,
                 eps=1e-6, pad=0, bias=True, mean=0.5, seed=0):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *n: torch.randn(*n, generator=gen, device="cuda")  # noqa: E731
        self.kw = dict(post=post, pre=pre, gate_act=gate_act, eps_post=eps, eps_pre=2 * eps, scale=scale, offset=offset)
        self.shape = BL.make_block_shape(D, post, pre, dtype, s_dtype, x_dtype, gate, gate_act, eps, 2 * eps, scale, offset)
        rows = lambda d, m: (normal(T + 1, D + pad) * 2 + m).to(dt(d))[:T, :D]  # noqa: E731
        self.y, self.r = rows(dtype, mean), rows(s_dtype, -mean)
        self.gate = {"none": None, "element": rows(dtype, 0), "token": normal(max(T, 1) * 3).to(dt(dtype))[:3 * T:3], "channel": normal(D)}[gate]
        norm = lambda kind: (None, None) if kind == "none" else (normal(D) * 0.3 + 1 - offset, normal(D) if bias and kind == "layer" else None)  # noqa: E731
        (self.w_post, self.b_post), (self.w_pre, self.b_pre) = norm(post), norm(pre)
        out = lambda d: torch.full((T + 1, D + pad), 77.0, device="cuda", dtype=dt(d))  # noqa: E731
        self.s_all, self.x_all = out(s_dtype), out(x_dtype)
        self.s, self.x = self.s_all[:T, :D], self.x_all[:T, :D] if pre != "none" else None

    def run(self, stream=None):
        BL.gdn_block_norm(self.shape, self.y, self.gate, self.w_post, self.b_post, self.r, self.w_pre, self.b_pre, self.s, self.x, stream)

    def check(self, rows=None):
        import torch
        torch.cuda.synchronize()
        pick = (lambda a: a) if rows is None else (lambda a: a if a is None else a[rows])
        gate = self.gate
        if gate is not None and gate.dim() == 1 and self.shape.gate == 2:
            gate = pick(gate[:, None])
        elif self.shape.gate == 1:
            gate = pick(gate)
        s, x = bo.block_norm(f64(pick(self.y)), f64(gate), f64(self.w_post), f64(self.b_post), f64(pick(self.r)), f64(self.w_pre), f64(self.b_pre), **self.kw)
        within(pick(self.s), *s)
        if x is not None:
            within(pick(self.x), *x)


def within(got, ref, bound):
    """|got - ref| <= bound, and 2^-8 of the value for the rounding to bf16."""
    import torch
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(ref) + bound) + 2.0 ** -134
    worst = np.abs(f64(got) - ref) - bound
    assert not np.isnan(worst).any() and worst.max(initial=-1.0) <= 0, float(worst.max())


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", [(1, 8), (1, 2048), (3, 64), (5, 504), (7, 520), (33, 1032), (2, 2056), (64, 2048), (9, 5120), (3, 8192), (2, 8200),
                                 (3, 16392), (1, 32768), (4099, 72), (4100, 2048), (4097, 1000)])
@pytest.mark.parametrize("post,pre", [("none", "rms"), ("layer", "layer"), ("rms", "layer"), ("rms", "none")])
def test_sizes_and_norms(T, D, post, pre):
    c = Call(T, D, post, pre, pad=8 * (D % 3), seed=T + D)
    c.run()
    c.check()
    assert (c.s_all[T:] == 77).all() and (c.s_all[:, D:] == 77).all()            # rows and columns beside the outputs
    assert (c.x_all[T:] == 77).all() and (c.x_all[:, D:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("s_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("x_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "element", "token", "channel"])
@pytest.mark.parametrize("gate_act", ["none", "sigmoid"])
def test_types_and_gates(dtype, s_dtype, x_dtype, gate, gate_act):
    for T, D, post in ((13, 776, "rms"), (5, 3000, "layer")):
        c = Call(T, D, post, "rms", dtype, s_dtype, x_dtype, gate, gate_act, scale=0.3, offset=1.0, pad=16, seed=D)
        c.run()
        c.check()


@pytest.mark.gpu
def test_a_mean_far_from_zero_and_a_large_eps():
    for mean, eps in ((300.0, 1e-6), (0.0, 10.0), (-50.0, 0.0)):
        c = Call(21, 2048, "layer", "layer", "f32", "f32", "f32", eps=eps, mean=mean)
        c.run()
        c.check()


@pytest.mark.gpu
def test_absent_parts():
    import torch
    for T, D in ((3, 2048), (5000, 512)):
        c = Call(T, D, "none", "rms")
        only = torch.empty_like(c.x)
        BL.gdn_block_norm(c.shape, None, None, None, None, c.r, c.w_pre, None, None, only)        # the norm by itself
        (s, es), (x, ex) = bo.block_norm(None, None, None, None, f64(c.r), f64(c.w_pre), None, **c.kw)
        torch.cuda.synchronize()
        within(only, x, ex)
        c.r = None                                                                                 # the first block: no stream yet
        c.run()
        (s, es), (x, ex) = bo.block_norm(f64(c.y), None, None, None, None, f64(c.w_pre), None, **c.kw)
        torch.cuda.synchronize()
        within(c.s, s, es)
        within(c.x, x, ex)


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", [(3, 2048), (4200, 1024)])
def test_in_place(T, D):
    """The stream over itself and x over the block's output give what separate outputs do; so does every output over every input."""
    import torch
    for s_over, x_over in (("r", "y"), ("y", "r"), ("r", None), (None, "gate")):
        c = Call(T, D, "rms", "layer", gate="element", gate_act="sigmoid", pad=8)
        c.run()
        torch.cuda.synchronize()
        want_s, want_x = c.s.clone(), c.x.clone()
        c.s = getattr(c, s_over) if s_over else c.s
        c.x = getattr(c, x_over) if x_over else c.x
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.s, want_s) and torch.equal(c.x, want_x)


@pytest.mark.gpu
def test_columns_of_one_buffer():
    """y, the stream and both outputs side by side in one wide buffer."""
    import torch
    c = Call(37, 256, "rms", "rms")
    c.run()
    wide = torch.zeros(37, 1024, dtype=torch.bfloat16, device="cuda")
    wide[:, :256], wide[:, 256:512] = c.y, c.r
    BL.gdn_block_norm(c.shape, wide[:, :256], None, c.w_post, None, wide[:, 256:512], c.w_pre, None, wide[:, 512:768], wide[:, 768:])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 512:768], c.s) and torch.equal(wide[:, 768:], c.x)


@pytest.mark.gpu
def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    for T, D in ((9, 2048), (4100, 512)):
        c = Call(T, D, "rms", "layer")
        c.run()
        torch.cuda.synchronize()
        want_s, want_x = c.s.clone(), c.x.clone()
        c.y[2, 5], c.r[4, 7] = float("nan"), float("inf")
        c.run()
        torch.cuda.synchronize()
        rest = [t for t in range(T) if t not in (2, 4)]
        assert torch.equal(c.s[rest], want_s[rest]) and torch.equal(c.x[rest], want_x[rest])
        assert c.s[2].isnan().all() and c.x[2].isnan().all()
        assert torch.isinf(c.s[4, 7]) and c.x[4].isnan().all()
        zero = Call(T, D, "rms", "rms")
        zero.y.zero_()
        zero.r.zero_()
        zero.run()
        torch.cuda.synchronize()
        assert (zero.s == 0).all() and (zero.x == 0).all()


@pytest.mark.gpu
def test_rows_whose_offsets_pass_32_bits():
    import torch
    T, D, wide = 70000, 64, 32768
    a, b = (torch.empty(T, wide, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Call(T, D, "rms", "rms")
    y, r, s, x = a[:, :D], a[:, D:2 * D], b[:, 64:64 + D], b[:, -D:]
    y.copy_(c.y)
    r.copy_(c.r)
    c.y, c.r, c.s, c.x = y, r, s, x
    c.run()
    c.check(slice(T - 300, T))
    c.check(slice(0, 300))


@pytest.mark.gpu
def test_another_stream_and_a_captured_graph():
    import torch
    c = Call(70, 2048, "rms", "rms", gate="token")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(side)
    side.synchronize()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for i in range(3):
        c.y.mul_(0.5).add_(i)
        c.s.zero_()
        graph.replay()
        c.check()
        got = c.s.clone(), c.x.clone()
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], c.s) and torch.equal(got[1], c.x)


def test_spans_past_63_bits_are_refused():
    assert raw(T=(1 << 31) - 1, ldy=1 << 32) == -11
    assert raw(T=(1 << 31) - 1, ldx=1 << 30) == -11
    assert raw(shaped(gate="token"), T=1 << 30, ldg=1 << 32) == -11


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", [(3, 8200), (300, 16384), (2, 16392), (300, 24584), (3, 32768)])
@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16")])
def test_in_place_of_wide_rows(T, D, types):
    """Rows of more than one piece to a thread: with four, the stream and the gate are read behind the first norm, between writes of outputs that lie over them."""
    import torch
    for s_over, x_over in (("r", "y"), ("y", "r"), ("r", None), (None, "gate"), ("gate", "r"), ("r", "gate")):
        c = Call(T, D, "rms", "layer", dtype=types[0], s_dtype=types[1], x_dtype=types[2], gate="element", gate_act="sigmoid", pad=8)
        of = {"y": types[0], "gate": types[0], "r": types[1], None: None}
        if of[s_over] not in (None, types[1]) or of[x_over] not in (None, types[2]):
            continue                                                  # (rows of another type cannot be the same)
        c.run()
        torch.cuda.synchronize()
        want_s, want_x = c.s.clone(), c.x.clone()
        c.s = getattr(c, s_over) if s_over else c.s
        c.x = getattr(c, x_over) if x_over else c.x
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.s, want_s) and torch.equal(c.x, want_x)
        if T < 10 and s_over == "r" and x_over == "y":
            c = Call(T, D, "rms", "layer", dtype=types[0], s_dtype=types[1], x_dtype=types[2], gate="element", gate_act="sigmoid", pad=8)
            c.run()
            c.check()
            assert torch.equal(c.s, want_s) and torch.equal(c.x, want_x)
