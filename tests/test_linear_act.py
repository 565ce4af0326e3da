"""Projections with an epilogue (gdn_linear_act, include/gdn_linear.h) against their oracle (the definition in fp64).

CPU part: oracle pins, refusals, the plan.  GPU part (marked gpu): element by element, every kernel that a plan can name.
Tolerance: the oracle's bound of fp32's error; one rounding more, 2^-8 of the value (half a step), for outputs in bf16.
"""
import numpy as np
import pytest

from oracle import linear_oracle as lo
from paper_2605_05219_amd import binding as B, linear as LN


# ----------------------------------------------------------------------------- the oracle
def test_oracle_hand_worked_case_and_known_values():
    x, w, up = np.array([[1.0, 2.0]]), np.array([[3.0, -1.0], [-1.0, 0.0]]), np.array([[0.0, 1.0], [2.0, 2.0]])
    y, _ = lo.linear_act(x, w, np.array([0.5, 0.0]), "relu", up, np.array([1.0, 0.0]), np.array([[10.0, 20.0]]), 2.0)
    assert np.array_equal(y, [[2 * 1.5 * 3 + 10, 20.0]])               # z = 1.5, -1; up = 3, 6
    assert np.array_equal(lo.linear_act(x, w, None, "relu2")[0], [[1.0, 0.0]])
    z = np.array([-1.0, 0.0, 1.0])
    assert np.allclose(lo.ACTS["gelu"](z), [-0.15865525393145707, 0, 0.8413447460685429])          # z Phi(z)
    assert np.allclose(lo.ACTS["gelu_tanh"](z), [-0.15880800939172324, 0, 0.8411919906082768])
    assert np.allclose(lo.ACTS["silu"](z), [-0.2689414213699951, 0, 0.7310585786300049]) and np.allclose(lo.ACTS["sigmoid"](z), [0.2689414213699951, 0.5, 0.7310585786300049])


def test_oracle_slopes_are_what_its_bound_takes_them_for():
    z = np.linspace(-20, 20, 400001)
    for act in ("silu", "gelu", "gelu_tanh"):
        assert np.abs(np.diff(lo.ACTS[act](z)) / np.diff(z)).max() <= 1.13
    assert np.abs(np.diff(lo.ACTS["sigmoid"](z)) / np.diff(z)).max() <= 0.25


# ----------------------------------------------------------------------------- refusals and the plan
def raw(epi=None, no_epilogue=False, **over):
    a = dict(x_ptr=0x100000, ldx=256, w_ptr=0x200000, ldw=256, bias_ptr=0x800000, y_ptr=0x400000, ldy=512, out_dtype=B.GDN_BF16, T=100, N=512, K=256)
    e = dict(act=1, res_dtype=B.GDN_BF16, scale=1.0, w_up=0x300000, ldw_up=256, bias_up=0x801000, residual=0x600000, ldr=512)
    a.update(over)
    e.update(epi or {})
    return LN.gdn_linear_act_raw(epilogue=None if no_epilogue else LN.gdn_linear_epilogue(**e), **a)


@pytest.mark.parametrize("epi,over,code", [
    ({}, dict(T=-1), -11), ({}, dict(N=-1), -11), ({}, dict(K=-64), -11), ({}, dict(out_dtype=7), -3), ({}, dict(K=200), -3), ({}, dict(K=0), -3),
    ({}, dict(ldx=128), -3), ({}, dict(ldw=192), -3), ({}, dict(ldy=256), -3), ({}, dict(x_ptr=0), -1), ({}, dict(w_ptr=0), -1), ({}, dict(y_ptr=0), -1),
    ({}, dict(x_ptr=0x100008), -2), ({}, dict(w_ptr=0x200004), -2), ({}, dict(y_ptr=0x400004), -2), ({}, dict(bias_ptr=0x800002), -2),
    ({}, dict(y_ptr=0x400008, out_dtype=B.GDN_F32), -2), ({}, dict(ldx=260), -2), ({}, dict(ldy=514), -2), ({}, dict(ldx=1 << 22), -11),
    (dict(act=7), {}, -3), (dict(act=-1), {}, -3), (dict(res_dtype=2), {}, -3), (dict(ldr=508), {}, -3), (dict(ldw_up=128), {}, -3),
    (dict(w_up=0), {}, -3),                                            # a bias of no product
    (dict(w_up=0x300008), {}, -2), (dict(ldw_up=260), {}, -2), (dict(bias_up=0x801001), {}, -2), (dict(residual=0x600004), {}, -2), (dict(ldr=514), {}, -2),
    (dict(residual=0x600008, res_dtype=B.GDN_F32), {}, -2), (dict(ldw_up=1 << 22), {}, -11), (dict(ldr=1 << 31), {}, -11), ({}, dict(ldy=1 << 31), -11),
    (dict(residual=0x400010), {}, -7), (dict(residual=0x400000, ldr=520), {}, -7), (dict(residual=0x400000, res_dtype=B.GDN_F32), {}, -7),
    ({}, dict(y_ptr=0x100000), -7), ({}, dict(y_ptr=0x200000), -7), ({}, dict(y_ptr=0x300000 - 512), -7), ({}, dict(y_ptr=0x800000), -7),
    ({}, dict(y_ptr=0x801000), -7),
])
def test_refusals(epi, over, code):
    assert raw(epi, **over) == code


def test_no_epilogue_and_empty_problems():
    assert raw(no_epilogue=True) == -1
    assert raw(T=0, x_ptr=0, y_ptr=0) == 0
    assert raw(N=0, w_ptr=0, y_ptr=0, ldy=0) == 0


def test_plan():
    rng = np.random.default_rng(9)
    for _ in range(300):
        T, N, K = int(np.exp(rng.uniform(0, 12))), int(np.exp(rng.uniform(0, 9.5))), 64 * int(rng.integers(1, 65))
        for gated in (False, True):
            shape, cols, rest = LN.gdn_linear_act_plan(T, N, K, gated)
            assert shape in (0, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11) and 0 < cols <= N and (shape < 6 or (T <= 1024 and cols == N))
            assert not (gated and (shape in (5, 6, 9) or rest == 5))
            if cols < N:
                assert shape == 2 and cols % (128 if gated else 256) == 0 and rest in (0, 3, 4, 5)
            if not gated and shape < 6:
                assert (shape, cols, rest) == LN.gdn_linear_plan(T, N, K)
    for knob in range(12):
        prev = LN.gdn_linear_act_tune(knob)
        try:
            assert LN.gdn_linear_act_plan(64, 512, 512, True)[:2] == ({1: 2, 5: 0, 6: 7, 9: 10}.get(knob, knob), 512)
            assert LN.gdn_linear_act_plan(64, 512, 512)[:2] == ({1: 2}.get(knob, knob), 512)
            assert LN.gdn_linear_act_plan(1025, 512, 512)[0] < 6
        finally:
            assert LN.gdn_linear_act_tune(prev) == knob
    assert LN.gdn_linear_act_tune(12) == -1
    for T, N, K, gated, code in [(0, 1, 64, 0, -11), (1, -1, 64, 0, -11), (1, 1, 0, 0, -11), (1, 1, 100, 0, -3), (1, 1, 64, 2, -3)]:
        with pytest.raises(B.GdnError) as ei:
            LN.gdn_linear_act_plan(T, N, K, gated)
        assert ei.value.code == code


def test_python_binding_refuses_mismatched_tensors():
    import torch
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16)  # noqa: E731
    good = dict(x=bf(4, 64), w=bf(8, 64), bias=torch.zeros(8), y=bf(4, 8), act="silu", w_up=bf(8, 64), bias_up=torch.zeros(8), residual=bf(4, 8))
    for over in (dict(w=bf(8, 128)), dict(y=bf(4, 9)), dict(x=torch.zeros(4, 64)), dict(bias=bf(8)), dict(bias=torch.zeros(7)), dict(w_up=bf(9, 64)),
                 dict(w_up=torch.zeros(8, 64)), dict(residual=bf(5, 8)), dict(residual=torch.zeros(4, 8, dtype=torch.float64)), dict(y=torch.zeros(4, 8, dtype=torch.float16)),
                 dict(act="swish"), dict(x=bf(4, 128)[:, ::2]), dict(bias_up=torch.zeros(16)[::2]), dict(y=bf(4, 16)[:, ::2]), dict(residual=bf(8, 4).t())):
        with pytest.raises(ValueError):
            LN.gdn_linear_act(**{**good, **over})
    with pytest.raises(B.GdnError) as ei:
        LN.gdn_linear_act(**{**good, "x": bf(64).expand(4, 64)})
    assert ei.value.code == -3


# ----------------------------------------------------------------------------- GPU
def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Call:
    def __init__(self, T, N, K, act="none", gated=False, bias=False, residual=None, out="bf16", scale=1.0, pad=0, seed=0):
        import torch
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *n: torch.randn(*n, generator=gen, device="cuda")  # noqa: E731
        up4 = lambda n: -(-n // 4) * 4  # noqa: E731
        self.x = normal(T, K + pad).bfloat16()[:, :K]
        weight = lambda: (normal(N, K + pad) * 2 * K ** -0.5).bfloat16()[:, :K]  # noqa: E731
        self.w, self.w_up = weight(), weight() if gated else None
        self.bias, self.bias_up = (normal(N) if bias else None), (normal(N) if bias and gated else None)
        self.residual = None if residual is None else normal(T, up4(N) + pad).to(dt[residual])[:, :N]
        self.all = torch.full((T + 2, up4(N) + 4 + pad), 77.0, device="cuda", dtype=dt[out])
        self.y, self.act, self.scale = self.all[:T, :N], act, scale

    def run(self, stream=None):
        LN.gdn_linear_act(self.x, self.w, self.bias, self.y, self.act, self.w_up, self.bias_up, self.residual, self.scale, stream)
        return self

    def check(self, rows=slice(None)):
        import torch
        torch.cuda.synchronize()
        res = None if self.residual is None else f64(self.residual[rows])
        ref, bound = lo.linear_act(f64(self.x[rows]), f64(self.w), f64(self.bias), self.act, f64(self.w_up), f64(self.bias_up), res, self.scale)
        if self.y.dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * (np.abs(ref) + bound) + 2.0 ** -134
        worst = np.abs(f64(self.y[rows]) - ref) - bound
        assert not np.isnan(worst).any() and worst.max(initial=-1.0) <= 0, float(worst.max())
        T, N = self.y.shape
        assert (self.all[T:] == 77).all() and (self.all[:, N:] == 77).all()       # what lies beside the outputs


@pytest.fixture
def knob():
    yield LN.gdn_linear_act_tune
    LN.gdn_linear_act_tune(-1)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 130, 1000])
@pytest.mark.parametrize("N,K", [(1, 64), (16, 128), (17, 576), (130, 1600), (515, 4096)])
@pytest.mark.parametrize("gated", [False, True])
def test_sizes(T, N, K, gated):
    Call(T, N, K, "silu" if gated else "none", gated, True, "bf16" if N % 2 else None, "bf16", pad=8 * (T % 3), seed=T * N).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("act", list(LN.ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T", [5, 100])
def test_activations_types_and_residuals(act, gated, T):
    for out in ("bf16", "f32"):
        for residual in (None, "bf16", "f32"):
            Call(T, 203, 320, act, gated, residual != "bf16", residual, out, -0.75, 16, seed=T).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [0, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_every_kernel(knob, shape, gated, out):
    """Each kernel on problems of one partial tile, of several with odd edges, and of few and many k steps."""
    for T, N, K, residual in ((3, 20, 64, "f32"), (64, 300, 192, None), (17, 71, 640, "bf16"), (128, 90, 1472, "f32"), (300, 523, 448, "bf16"), (517, 777, 64, "f32")):
        knob(shape)
        Call(T, N, K, "gelu_tanh", gated, True, residual, out, 0.5, 8, seed=N).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("T,N,K,gated", [(3000, 5300, 192, False), (3000, 2650, 192, True), (6000, 6144, 128, False), (8192, 2080, 128, True)])
def test_large_problems_and_cut_columns(T, N, K, gated):
    c = Call(T, N, K, "silu", gated, True, "bf16", "bf16", seed=1).run()
    for rows in (slice(0, 200), slice(T // 2, T // 2 + 150), slice(T - 130, T)):
        c.check(rows)


@pytest.mark.gpu
def test_some_of_these_problems_are_cut():
    cut = [LN.gdn_linear_act_plan(T, N, 2048, g)[1] < N for T, N, g in ((8192, 8224, False), (8192, 4112, True), (2048, 4112, True))]
    assert all(cut)
    c = Call(2048, 4112, 2048, "silu", True, True, "f32", "f32", seed=2).run()
    for rows in (slice(0, 40), slice(2020, 2048)):
        c.check(rows)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_residual_in_place(T, dtype):
    import torch
    c = Call(T, 333, 256, "silu", True, True, dtype, dtype, 0.5).run()
    torch.cuda.synchronize()
    want = c.y.clone()
    c.y = c.residual
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [9, 200])
def test_values_that_are_not_finite_stay_in_their_row(T):
    """A NaN or an infinity in a row of x reaches that row's outputs and no other; one in a row of w its output column and no other."""
    import torch
    c = Call(T, 150, 256, "relu", True).run()
    torch.cuda.synchronize()
    want = c.y.clone()
    c.x[3, 70], c.x[5, 1] = float("nan"), float("inf")
    c.w[7, 3] = float("nan")
    c.run()
    torch.cuda.synchronize()
    keep = torch.ones(T, 150, dtype=torch.bool, device="cuda")
    keep[[3, 5]] = False
    keep[:, 7] = False
    assert torch.equal(c.y[keep], want[keep]) and c.y[3].isnan().all() and c.y[:, 7].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", list(LN.ACTS))
@pytest.mark.parametrize("T", [3, 200])
def test_activations_at_their_ends(act, T):
    """Sums of zero, of either sign far out, and infinite: what the formula's limits are (an infinity times zero is NaN)."""
    import torch
    K, N = 64, 8                                                      # (rows of y are whole groups of four)
    x, w = torch.zeros(T, K, device="cuda", dtype=torch.bfloat16), torch.zeros(N, K, device="cuda", dtype=torch.bfloat16)
    x[:, 0] = 1
    z = [0.0, 50.0, -50.0, 1e30, -1e30, float("inf"), 1.0, -1.0]
    w[:, 0] = torch.tensor(z, device="cuda")
    x[:, 1:], w[:, 1:] = 0, 0
    y = torch.empty(T, N, device="cuda")
    LN.gdn_linear_act(x, w, None, y, act)
    zb = w[:, 0].double()
    with np.errstate(all="ignore"):
        want = {"none": zb, "silu": torch.nn.functional.silu(zb), "gelu": torch.nn.functional.gelu(zb), "gelu_tanh": torch.nn.functional.gelu(zb, approximate="tanh"),
                "relu": torch.relu(zb), "relu2": torch.relu(zb) ** 2, "sigmoid": torch.sigmoid(zb)}[act].float()
    torch.cuda.synchronize()
    assert torch.allclose(y, want.expand(T, N), rtol=1e-5, atol=1e-12, equal_nan=True), (y[0], want)


@pytest.mark.gpu
def test_rows_whose_offsets_pass_32_bits():
    import torch
    T, wide = 70000, 32768
    x, y = (torch.empty(T, wide, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Call(T, 72, 64, "silu", True)
    x[:, :64].copy_(c.x)
    c.x, c.residual, c.y = x[:, :64], x[:, 64:136], y[:, -72:]
    c.residual.copy_(torch.randn(T, 72, device="cuda"))
    c.all = c.y
    c.run()
    torch.cuda.synchronize()
    for rows in (slice(0, 100), slice(T - 100, T)):
        ref, bound = lo.linear_act(f64(c.x[rows]), f64(c.w), None, "silu", f64(c.w_up), None, f64(c.residual[rows]))
        assert (np.abs(f64(c.y[rows]) - ref) <= bound + 2.0 ** -8 * (np.abs(ref) + bound)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 64, 500])
def test_another_stream_and_a_captured_graph(T):
    import torch
    c = Call(T, 520, 512, "silu", True, True, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(side)
    side.synchronize()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for i in range(3):
        c.x.mul_(0.5).add_(0.1 * i)
        c.y.zero_()
        graph.replay()
        c.check()
        got = c.y.clone()
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(got, c.y)


def test_spans_past_63_bits_and_more_outputs_than_threads_are_refused():
    assert raw(T=1 << 37, N=64, ldy=1 << 24) == -11
    assert raw(dict(ldr=1 << 24), T=1 << 37, N=64) == -11
    assert raw(dict(ldw_up=1 << 60)) == -11
    assert raw(dict(ldr=1 << 24), N=1 << 24, ldy=1 << 24) == -11


def test_kernels_of_few_rows_keep_to_the_threads_of_a_launch():
    for knob in range(6, 12):
        prev = LN.gdn_linear_act_tune(knob)
        try:
            for gated in (False, True):
                assert LN.gdn_linear_act_plan(1024, (1 << 24) - 1, 64, gated)[0] < 6
                assert LN.gdn_linear_act_plan(16, 1 << 20, 64, gated)[0] >= 6
        finally:
            LN.gdn_linear_act_tune(prev)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
@pytest.mark.parametrize("T", [3, 200])
def test_activations_keep_their_digits_far_out(act, T):
    """Values that are small because z is far below zero are right to a relative error: of an exponential (its argument + 4) 2^-23, twice that for the roundings of its
    argument, 8 units for the sums, products, reciprocals and polynomials around it; and what lies below the least normal number may be zero."""
    import torch
    from scipy.special import erfc
    far = {"gelu": 13.0, "gelu_tanh": 9.0}.get(act, 80.0)
    z = -torch.exp(torch.linspace(np.log(2.0 ** -7), np.log(far), 800, device="cuda", dtype=torch.float64)).bfloat16()
    K, N = 64, z.numel()
    x, w = torch.zeros(T, K, device="cuda", dtype=torch.bfloat16), torch.zeros(N, K, device="cuda", dtype=torch.bfloat16)
    x[:, 0], w[:, 0] = 1, z
    y = torch.empty(T, N, device="cuda")
    LN.gdn_linear_act(x, w, None, y, act)
    z = f64(z)
    u2 = np.sqrt(8 / np.pi) * (z + 0.044715 * z ** 3)
    with np.errstate(over="ignore"):                                  # (of the activations that are not looked at)
        want = {"silu": z / (1 + np.exp(-z)), "gelu": 0.5 * z * erfc(-z / np.sqrt(2)), "gelu_tanh": z / (1 + np.exp(-u2)), "sigmoid": 1 / (1 + np.exp(-z))}[act]
    arg = {"gelu": z * z / 2, "gelu_tanh": np.abs(u2)}.get(act, np.abs(z))
    torch.cuda.synchronize()
    worst = np.abs(f64(y) - want) - ((2 * (arg + 4) + 8) * 2.0 ** -23 * np.abs(want) + 2.0 ** -126 * np.maximum(1, np.abs(z)))
    assert worst.max() <= 0, [(float(z[n]), float(y[t, n]), float(want[n])) for t, n in [np.unravel_index(int(worst.argmax()), worst.shape)]]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [-1, 0, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11])
@pytest.mark.parametrize("T,N,K", [(5, 50, 8192), (37, 17, 4160), (70, 73, 4096), (33, 9, 6144)])
@pytest.mark.parametrize("gated", [False, True])
def test_every_term_of_a_long_sum_counts(knob, shape, T, N, K, gated):
    """Small whole numbers, whose products and sums fp32 holds exactly in any order: the outputs are equal, so no term is lost or taken twice."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(K + N)
    whole = lambda *n: torch.randint(-2, 3, n, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, behind = whole(T, K), torch.full((N + 40, K), float("nan"), dtype=torch.bfloat16, device="cuda")
    w, up = behind.clone()[:N], behind.clone()[:N]                    # (what lies behind a weight's last row counts for nothing)
    w.copy_(whole(N, K))
    up.copy_(whole(N, K))
    res = torch.zeros(T, -(-N // 4) * 4, device="cuda")[:, :N]
    res.copy_(torch.randint(-1000, 1000, (T, N), generator=gen, device="cuda"))
    bias = torch.randint(-9, 9, (N,), generator=gen, device="cuda").float()
    y = torch.full((T, -(-N // 4) * 4), 77.0, device="cuda")[:, :N]
    knob(shape)
    LN.gdn_linear_act(x, w, bias, y, "none", up if gated else None, None, res, 0.5)
    z = f64(x) @ f64(w).T + f64(bias)
    want = 0.5 * z * (f64(x) @ f64(up).T if gated else 1.0) + f64(res)
    assert np.abs(f64(x)).sum(1).max() * 2 < 2 ** 24 and np.abs(2 * want).max() + 2000 < 2 ** 24      # exact in fp32, in halves too
    torch.cuda.synchronize()
    assert np.array_equal(f64(y), want)
