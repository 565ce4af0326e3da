"""The mixture of experts (include/gdn_moe.h) against its oracle (the definition in fp64, with a bound of fp32's error).

CPU part: oracle pins, exports, refusals (every check returns before a pointer is used).  GPU part (marked gpu): choices exactly, weights and
outputs element by element.  Tolerance: the oracle's bound, and 2^-8 of the value (half a step of bf16) for y.
"""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import linear_oracle as lo, moe_oracle as mo
from paper_2605_05219_amd import binding as B, moe as MO

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ----------------------------------------------------------------------------- the oracle
def test_oracle_hand_worked_case():
    x = np.array([[1.0, 2.0]])
    wr = np.array([[0.0, 0.0], [1.0, 0.0], [0.0, 0.5]])                # logits 0, 1, 1: the lower index first
    gu = np.zeros((3, 2, 2))
    gu[1], gu[2] = [[1, 1], [0, 1]], [[2, 0], [1, 0]]                  # gate 3, up 2 -> 6;  gate 2, up 1 -> 2
    down = np.array([[[9.0], [9.0]], [[1.0], [0.0]], [[1.0], [4.0]]])
    ids, (p, _), (y, _) = mo.moe(x, wr, None, gu, down, np.array([[10.0, 20.0]]), 2, "relu")
    assert ids.tolist() == [[1, 2]] and p.tolist() == [[0.5, 0.5]]
    assert y.tolist() == [[10 + 3 + 1, 20 + 4]]
    ids, (p, _), _ = mo.moe(x, wr, np.array([2.0, 0.0, -np.inf]), gu, down, None, 3, "relu", "sigmoid", False, 2.0)
    s1 = 1 / (1 + np.exp(-1.0))
    assert ids.tolist() == [[0, 1, -1]] and np.allclose(p, [[1.0, 2 * s1, 0]])
    ids, (p, _), _ = mo.moe(x, wr, None, gu, down, None, 1, "relu", "softmax", False)
    assert np.allclose(p, np.e / (1 + 2 * np.e))


def test_oracle_one_expert_is_the_plain_gated_block():
    rng = np.random.default_rng(0)
    x, gu, down = rng.standard_normal((5, 8)), rng.standard_normal((1, 12, 8)), rng.standard_normal((1, 8, 6))
    _, _, (y, _) = mo.moe(x, rng.standard_normal((1, 8)), None, gu, down, None, 1)
    h = mo.to_bf16(lo.ACTS["silu"](x @ gu[0, :6].T) * (x @ gu[0, 6:].T))
    assert np.allclose(y, h @ down[0].T)


def test_oracle_bf16_rounding():
    import torch
    a = np.concatenate([np.random.default_rng(1).standard_normal(2000) * 10.0 ** np.arange(2000).clip(0, 30), [0.0, -0.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, np.inf]])
    a = a.astype(np.float32)
    assert np.array_equal(mo.to_bf16(a), torch.from_numpy(a).bfloat16().double().numpy())


# ----------------------------------------------------------------------------- refusals
def test_library_exports_every_symbol_the_moe_header_declares():
    header = open(os.path.join(ROOT, "include", "gdn_moe.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(gdn_moe\w*)\s*\(", header))
    assert declared == set(MO.EXPORTS)
    L = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert getattr(L, name) is not None


def altered(**fields):
    s = MO.make_moe_shape(8, 2, 256, 128)
    for name, v in fields.items():
        setattr(s, name, v)
    return s


def raw(shape=None, **over):
    shape = altered() if shape is None else shape
    a = dict(x=0x100000, ldx=256, w_router=0x200000, choice_bias=0x300000, w_gate_up=0x1000000, w_down=0x2000000, add=0x400000, ld_add=256, y=0x500000, ldy=256,
             ids=0x600000, weights=0x700000, T=10, workspace=0x4000000, workspace_bytes=1 << 24)
    a.update(over)
    return MO.gdn_moe_raw(shape, **a)


@pytest.mark.parametrize("shape,over,code", [
    (altered(E=0), {}, -3), (altered(E=1025), {}, -3), (altered(k=0), {}, -3), (altered(k=9), {}, -3), (altered(E=64, k=17), {}, -3),
    (altered(D=96), {}, -3), (altered(F=0), {}, -3), (altered(F=65), {}, -3), (altered(D=32832), {}, -3), (altered(act=7), {}, -3), (altered(act=-1), {}, -3),
    (altered(score=2), {}, -3), (altered(normalise=2), {}, -3), (altered(router_dtype=3), {}, -3), (altered(routed_scale=float("nan")), {}, -3),
    (None, dict(T=-1), -11), (None, dict(T=1 << 23), -11), (None, dict(T=1 << 40), -11), (None, dict(ldx=1 << 31), -11), (None, dict(ldy=1 << 31), -11),
    (None, dict(ldx=1 << 28), -11), (altered(F=32768), dict(T=20000, workspace_bytes=1 << 40), -11),
    (None, dict(x=0), -1), (None, dict(w_router=0), -1), (None, dict(w_gate_up=0), -1), (None, dict(w_down=0), -1), (None, dict(y=0), -1),
    (None, dict(ldx=248), -3), (None, dict(ldy=0), -3), (None, dict(ld_add=-256), -3),
    (None, dict(ldx=260), -2), (None, dict(ldy=257), -2), (None, dict(ld_add=258), -2), (None, dict(x=0x100008), -2), (None, dict(y=0x500002), -2), (None, dict(add=0x400004), -2),
    (None, dict(w_router=0x200008), -2), (None, dict(w_gate_up=0x1000002), -2), (None, dict(w_down=0x2000008), -2), (None, dict(choice_bias=0x300002), -2),
    (None, dict(ids=0x600001), -2), (None, dict(weights=0x700002), -2),
    (None, dict(workspace=0), -9), (None, dict(workspace=0x4000008), -9), (None, dict(workspace_bytes=1000), -9),
    (None, dict(y=0x100000), -7),                                  # the router has read x, the experts have not
    (None, dict(y=0x400000, ldy=264), -7), (None, dict(y=0x400010), -7), (None, dict(ids=0x500000), -7), (None, dict(weights=0x600000), -7),
    (None, dict(ids=0x300000), -7), (None, dict(weights=0x200000), -7), (None, dict(y=0x4000000), -7), (None, dict(x=0x4000100), -7), (None, dict(y=0x2000000), -7),
    (None, dict(y=0x1000000 - 512), -7),
])
def test_refusals(shape, over, code):
    assert raw(shape, **over) == code


def test_no_shape_and_no_tokens():
    assert MO.gdn_moe_raw(None) == -1
    assert raw(T=0, x=0, y=0, workspace=0) == 0
    assert MO.gdn_moe_workspace_bytes(altered(), 0) > 0
    sizes = [MO.gdn_moe_workspace_bytes(altered(), T) for T in (1, 2, 100, 5000)]
    assert sizes == sorted(sizes)
    with pytest.raises(B.GdnError):
        MO.gdn_moe_workspace_bytes(altered(k=9), 1)


def test_python_binding_refuses_mismatched_tensors():
    import torch
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16)  # noqa: E731
    shape = MO.make_moe_shape(8, 2, 128, 64)
    good = dict(x=bf(4, 128), w_router=bf(8, 128), choice_bias=torch.zeros(8), w_gate_up=bf(8, 128, 128), w_down=bf(8, 128, 64), add=None, y=bf(4, 128),
                ids=torch.zeros(4, 2, dtype=torch.int32), weights=torch.zeros(4, 2), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    for over in (dict(x=bf(4, 64)), dict(y=bf(5, 128)), dict(add=bf(4, 64)), dict(x=torch.zeros(4, 128)), dict(w_router=torch.zeros(8, 128)), dict(w_router=bf(7, 128)),
                 dict(choice_bias=bf(8)), dict(w_gate_up=bf(8, 64, 128)), dict(w_gate_up=bf(8, 128, 256)[:, :, ::2]), dict(w_down=bf(8, 64, 128)), dict(ids=torch.zeros(4, 2)),
                 dict(ids=torch.zeros(4, 3, dtype=torch.int32)), dict(weights=torch.zeros(2, 4).t()), dict(workspace=torch.zeros(1 << 21, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            MO.gdn_moe(shape, **{**good, **over})
    with pytest.raises(B.GdnError) as ei:
        MO.gdn_moe(shape, **{**good, "workspace": None})
    assert ei.value.code == -9
    with pytest.raises(B.GdnError) as ei:
        MO.gdn_moe(shape, **{**good, "add": bf(128).expand(4, 128)})
    assert ei.value.code == -3


# ----------------------------------------------------------------------------- GPU
def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


class Call:
    def __init__(self, T, E, k, D, F, act="silu", score="softmax", normalise=True, scale=1.0, router="bf16", bias=None, add=False, pad=0, seed=0, sharp=1.5):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *n, s=1.0: torch.randn(*n, generator=gen, device="cuda") * s  # noqa: E731
        self.kw = dict(act=act, score=score, normalise=normalise, routed_scale=scale)
        self.shape = MO.make_moe_shape(E, k, D, F, router_dtype=router, **self.kw)
        rows = lambda: normal(T, D + pad).bfloat16()[:, :D]  # noqa: E731
        self.x, self.add = rows(), rows() if add else None
        self.wr = normal(E, D, s=sharp * D ** -0.5).to(torch.float32 if router == "f32" else torch.bfloat16)
        self.bias = None if bias is None else torch.as_tensor(bias, dtype=torch.float32).cuda() if not isinstance(bias, bool) else normal(E, s=0.1)
        self.gu, self.down = normal(E, 2 * F, D, s=D ** -0.5).bfloat16(), normal(E, D, F, s=F ** -0.5).bfloat16()
        self.all = torch.full((T + 1, D + pad), 77.0, device="cuda", dtype=torch.bfloat16)
        self.y = self.all[:T, :D]
        self.ids = torch.full((T, k), -5, device="cuda", dtype=torch.int32)
        self.weights = torch.full((T, k), -5.0, device="cuda")
        self.ws = torch.full((MO.gdn_moe_workspace_bytes(self.shape, T),), 255, device="cuda", dtype=torch.uint8)      # NaNs and -1
        self.k = k

    def run(self, stream=None):
        MO.gdn_moe(self.shape, self.x, self.wr, self.bias, self.gu, self.down, self.add, self.y, self.ids, self.weights, self.ws, stream)
        return self

    def reference(self):
        return mo.moe(f64(self.x), f64(self.wr), f64(self.bias), f64(self.gu), f64(self.down), f64(self.add), self.k, **self.kw)

    def check(self, ref=None):
        import torch
        torch.cuda.synchronize()
        ids, (p, ep), (y, ey) = self.reference() if ref is None else ref
        assert np.array_equal(self.ids.cpu().numpy(), ids)
        assert (np.abs(f64(self.weights) - p) <= ep).all()
        got = f64(self.y)
        worst = np.abs(got - y) - (ey + 2.0 ** -8 * (np.abs(y) + ey) + 2.0 ** -134)
        assert not np.isnan(worst).any() and worst.max(initial=-1.0) <= 0, float(worst.max())
        T, D = self.y.shape
        assert (self.all[T:] == 77).all() and (self.all[:, D:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 16, 17, 40, 65, 130])
@pytest.mark.parametrize("E,k,D,F", [(8, 2, 128, 64), (60, 4, 320, 192), (64, 6, 512, 128), (130, 10, 256, 64), (1, 1, 64, 128)])
def test_sizes(T, E, k, D, F):
    Call(T, E, k, D, F, pad=8 * (T % 3), add=bool(T % 2), seed=T + E).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("E,k,T", [(512, 16, 30), (1000, 10, 9), (1024, 1, 70), (16, 16, 50), (3, 2, 300)])
def test_many_experts_and_choices(E, k, T):
    Call(T, E, k, 128, 64, seed=E).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("router", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [None, True])
def test_scores(score, normalise, router, bias):
    for T, act in ((3, "gelu"), (50, "silu"), (150, "relu2")):
        Call(T, 32, 5, 192, 128, act, score, normalise, 2.5 if score == "sigmoid" else 1.0, router, bias, seed=T).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 20, 200])
def test_an_uneven_choice(T):
    """Every token to the same experts, by their bias: one has all rows, most none."""
    bias = np.zeros(64)
    bias[[63, 5, 17]] = 50, 40, 30
    c = Call(T, 64, 4, 256, 128, bias=bias, seed=3).run()
    c.check()
    assert (c.ids[:, :3].cpu().numpy() == [63, 5, 17]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 30])
def test_equal_keys_go_to_the_lowest_index(T):
    c = Call(T, 96, 6, 128, 64, seed=4)
    c.wr[50:] = c.wr[10]                                              # 47 equal experts among 96 (the 10th with them)
    c.wr[0:4] = 0
    c.wr[1] = -c.wr[1]                                                # a sum of -0 is a sum of 0
    c.run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [False, True])
def test_masked_experts(score, normalise):
    """A bias of -infinity keeps experts from being chosen, down to fewer than k and to none."""
    for left in (7, 2, 1, 0):
        bias = np.full(40, -np.inf)
        bias[[3, 11, 12, 20, 29, 38, 39][:left]] = 0
        for T in (1, 35):
            for add in (False, True):
                c = Call(T, 40, 4, 128, 64, "silu", score, normalise, 1.5, bias=bias, add=add, seed=left)
                c.gu[0], c.down[1] = float("nan"), float("inf")       # of experts that are not chosen
                c.run().check()
                if left < 4:
                    assert (c.ids[:, left:] == -1).all() and (c.weights[:, left:] == 0).all()


@pytest.mark.gpu
def test_a_weight_of_zero_leaves_its_expert_out():
    """Scores that underflow: the choice stands, what its expert gives does not reach the sum."""
    c = Call(5, 8, 3, 64, 64, score="sigmoid", normalise=False)
    c.x[:] = 1
    c.wr[:] = -64                                                     # logits of -4096
    c.wr[2] = 0
    c.gu[0] = float("inf")
    c.run()
    ids, (p, ep), (y, ey) = c.reference()
    assert ids.tolist() == [[2, 0, 1]] * 5 and (p == [0.5, 0, 0]).all()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4, 70])
@pytest.mark.parametrize("score,normalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_a_token_that_is_not_finite_keeps_to_itself(T, score, normalise):
    import torch
    c = Call(T, 32, 4, 128, 64, "silu", score, normalise, seed=6, add=True).run()
    torch.cuda.synchronize()
    want = c.y.clone(), c.ids.clone(), c.weights.clone()
    c.x[1, 9] = float("nan")
    c.x[2] = float("inf")                                             # logits of either infinity and NaN
    c.run()
    torch.cuda.synchronize()
    rest = [t for t in range(T) if t not in (1, 2)]
    for got, before in zip((c.y, c.ids, c.weights), want):
        assert torch.equal(got[rest], before[rest])
    assert c.y[1].isnan().all() and c.weights[1].isnan().all() and c.ids[1].tolist() == [0, 1, 2, 3]
    assert c.y[2].isnan().all()
    ids = c.ids[2].tolist()
    assert len(set(ids)) == 4 and all(0 <= e < 32 for e in ids)


@pytest.mark.gpu
def test_absent_outputs_and_y_over_add():
    import torch
    for T in (1, 60):
        c = Call(T, 24, 3, 192, 64, add=True, pad=8, seed=8).run()
        c.check()
        want = c.y.clone()
        c.ids = c.weights = None
        c.y = c.add
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 33, 257])
def test_the_same_call_gives_the_same_bits(T):
    """Whatever order the choices of an expert are listed in, and whatever the workspace held."""
    import torch
    c = Call(T, 16, 4, 256, 128, seed=9).run()
    torch.cuda.synchronize()
    want = c.y.clone()
    for fill in (0, 127, 255):
        c.ws.fill_(fill)
        c.y.zero_()
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 64])
def test_another_stream_and_captured_graphs_with_one_workspace(T):
    import torch
    c = Call(T, 48, 4, 256, 128, seed=10, bias=True, score="sigmoid")
    d = Call(T, 48, 4, 256, 128, seed=11)
    d.ws = c.ws                                                       # one after the other on one stream
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(side)
    d.run(side)
    side.synchronize()
    c.check()
    d.check()
    graphs = []
    for call in (c, d):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call.run()
    for i in range(3):
        for call in (c, d):
            call.x.mul_(-1.5 if i == 1 else 0.5)
            call.y.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for call in (c, d):
            call.check()
            got = call.y.clone()
            call.run()
            torch.cuda.synchronize()
            assert torch.equal(got, call.y)


@pytest.fixture
def knob():
    yield MO.gdn_moe_tune
    MO.gdn_moe_tune(-1)


def test_knob_round_trip(knob):
    assert [knob(v) for v in (0, 2, 3, 6, 1, 2, 9)] == [-1, 0, 2, 3, 6, -1, 2]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [0, 2, 3, 6])
@pytest.mark.parametrize("T,E,k,D,F,bias", [(1, 8, 2, 64, 64, None), (3, 600, 5, 128, 64, None), (30, 60, 4, 320, 192, None), (32, 300, 16, 4160, 64, None), (700, 8, 3, 256, 320, None),
                                            (300, 20, 4, 128, 64, "one"), (90, 130, 10, 192, 128, None), (80, 12, 3, 1088, 1152, None)])
def test_every_kernel(knob, shape, T, E, k, D, F, bias):
    """The tiles on experts of no row, of part of a tile and of several, and where all tokens take the same ones; the kernels of few tokens up to their most."""
    if shape == 6 and T > 32:
        pytest.skip("few tokens are at most 32")
    if bias:
        bias = np.zeros(E)
        bias[[2, E - 1]] = 50
    knob(shape)
    Call(T, E, k, D, F, "gelu_tanh", bias=bias, add=True, pad=8, seed=T).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [3, 6])
@pytest.mark.parametrize("T", [1, 7])
def test_masks_and_zero_weights_in_every_path(knob, shape, T):
    """Fewer than k choices, none, and a weight of zero in front of and between choices that count."""
    knob(shape)
    for left in (0, 1, 3):
        bias = np.full(70, -np.inf)
        bias[[3, 11, 69][:left]] = 0
        c = Call(T, 70, 4, 128, 128, "silu", "sigmoid", False, 1.5, bias=bias, add=True, seed=left)
        c.gu[0] = float("nan")
        c.run().check()
    c = Call(T, 12, 4, 64, 64, score="sigmoid", normalise=False, bias=np.array([3.0, 0, 2, 0, 1, 0, 0, 0, 0, 0, 0, 0.5]))
    c.x[:] = 1
    c.wr[[0, 4]] = -64                                                # chosen by their bias, weights that underflow
    c.gu[0] = c.down[4] = float("inf")
    c.run().check()
    assert c.ids[0, :3].tolist() == [0, 2, 4] and c.weights[0, 0] == 0 and c.weights[0, 2] == 0


@pytest.mark.gpu
def test_more_tokens_than_a_grid_has_rows():
    import torch
    T = 16 * 65536 + 5
    c = Call(T, 3, 1, 64, 64, add=True, seed=5).run()
    torch.cuda.synchronize()
    some = torch.cat([torch.arange(40), torch.arange(65520, 65560), torch.arange(T - 40, T)]).cuda()
    ids, (p, ep), (y, ey) = mo.moe(f64(c.x[some]), f64(c.wr), None, f64(c.gu), f64(c.down), f64(c.add[some]), 1, **c.kw)
    assert np.array_equal(c.ids[some].cpu().numpy(), ids) and (np.abs(f64(c.weights[some]) - p) <= ep).all()
    worst = np.abs(f64(c.y[some]) - y) - (ey + 2.0 ** -8 * (np.abs(y) + ey) + 2.0 ** -134)
    assert not np.isnan(worst).any() and worst.max() <= 0, float(worst.max())
    assert (c.all[T:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("E", [60, 100, 200, 400, 1000])
@pytest.mark.parametrize("T,F", [(9, 64), (25, 64), (25, 192), (32, 320)])
def test_few_tokens_on_few_and_many_workgroups(knob, E, T, F):
    """The kernels of few tokens whose first product has fewer workgroups than the chip, about as many, and more, with every number of experts to a lane."""
    knob(6)
    bias = np.zeros(E)
    bias[E // 2] = 20                                                 # one that all tokens take
    Call(T, E, 4, 192, F, "silu", "sigmoid", True, 2.0, router="f32", bias=bias, add=bool(T % 2), pad=8, seed=E).run().check()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [-1, 0, 2, 3, 6])
@pytest.mark.parametrize("T,E,k,D,F", [(8, 16, 4, 2048, 128), (24, 8, 3, 1024, 64), (31, 40, 8, 576, 192)])
def test_a_row_is_the_same_wherever_its_token_stands(knob, shape, T, E, k, D, F):
    """Equal tokens of one call give equal bits, and so does each token of a batch in another order (T, E, k, D and F choose the kernels; they are the same)."""
    import torch
    knob(shape)
    c = Call(T, E, k, D, F, seed=T)
    c.x[T // 2:2 * (T // 2)] = c.x[:T // 2]
    c.run()
    torch.cuda.synchronize()
    half = T // 2
    assert torch.equal(c.ids[:half], c.ids[half:2 * half]) and torch.equal(c.weights[:half], c.weights[half:2 * half])
    assert torch.equal(c.y[:half], c.y[half:2 * half])
    want = c.y.clone()
    order = torch.randperm(T, generator=torch.Generator().manual_seed(T)).cuda()
    c.x.copy_(c.x[order])
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.y, want[order])
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 50])
@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("logits", [[-95, -90, -96, -103, -91, -94, -89, -92],      # sigmoids between 2^-149 and 2^-126
                                    [-200, -203, -201, -202, -207, -204, -206, -205],      # keys of zero: the lowest indices
                                    [-800, -801, -799, -802, -750, -740, -700, -900], [-60, -100, -63.5, -65, -64.5, -88, -200, -300], [-70, 3, -90, -1, -66, -68, -120, -100],
                                    [float("-inf")] * 8, [-120, float("-inf"), -121, float("-inf"), -122, -123, -124, -125]])
def test_sigmoids_of_far_logits(T, normalise, logits):
    """Weights that are divided by their sum are what they are however small the sigmoids, also below the least number of fp32."""
    import torch
    c = Call(T, 8, 3, 64, 64, score="sigmoid", normalise=normalise, scale=2.5, add=True, seed=1)
    c.x[:, 1:], c.x[:, 0] = 0, 1
    c.wr[:, 1:], c.wr[:, 0] = 0, torch.tensor(logits, device="cuda")
    c.run().check()
    if normalise and logits[0] != float("-inf"):
        assert abs(float(c.weights[0].sum()) - 2.5) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [-1, 0, 2, 3, 6])
@pytest.mark.parametrize("T,E,k,D,F", [(1, 8, 4, 2048, 1088), (30, 6, 1, 4096, 576), (30, 5, 4, 1088, 2048), (200, 4, 2, 2048, 1024), (700, 6, 1, 576, 4096)])
def test_every_term_of_the_sums_counts(knob, shape, T, E, k, D, F):
    """Small whole numbers: the first products are exact in fp32 in any order, h is rounded where the definition rounds it, and the second products and the sum of the choices, of
    weights that are powers of two, are exact again.  So y is equal to the last bit, and no term is lost or taken twice."""
    import torch
    if shape == 6 and T > 32:
        pytest.skip("few tokens are at most 32")
    knob(shape)
    c = Call(T, E, k, D, F, "none", add=True, seed=D)
    gen = torch.Generator(device="cuda").manual_seed(T)
    whole = lambda t: t.copy_(torch.randint(-1, 2, t.shape, generator=gen, device="cuda"))  # noqa: E731
    for t in (c.x, c.gu, c.down):
        whole(t)
    c.add.copy_(torch.randint(-100, 100, c.add.shape, generator=gen, device="cuda"))
    if k > 1:
        c.wr.zero_()                                                  # equal keys: the first k, 1 / k each
    c.run()
    torch.cuda.synchronize()
    ids, p, _ = mo.route(f64(c.x), f64(c.wr), None, k)
    assert np.array_equal(c.ids.cpu().numpy(), ids) and np.array_equal(f64(c.weights), np.full((T, k), 1.0 / k)) and np.allclose(p, 1.0 / k)
    x, gu, down, want, size = f64(c.x), f64(c.gu), f64(c.down), f64(c.add), np.abs(f64(c.add))
    for e in range(E):
        t = np.nonzero((ids == e).any(1))[0]
        g, u = x[t] @ gu[e, :F].T, x[t] @ gu[e, F:].T
        assert not t.size or (np.abs(g).max() < 2 ** 12 and np.abs(u).max() < 2 ** 12)
        h = mo.to_bf16(g * u / k)
        want[t] += h @ down[e].T
        size[t] += np.abs(h) @ np.abs(down[e]).T
    assert size.max() * k < 2 ** 24                                  # (in units of 1 / k)
    assert np.array_equal(f64(c.y), mo.to_bf16(want))
