"""The residual stream's norm, the projections with their epilogues and the mixture of experts together, as a layer's feed-forward half uses them.

Every tensor of a step is held against the operator's oracle on what the step itself made before it (its buffers hold that), with the oracle's bound and,
for tensors in bf16, half a step, 2^-8 of the value.  So each operator is right on what the others give it, and gets what it should."""
import numpy as np
import pytest

from oracle import block_oracle as bo, linear_oracle as lo, moe_oracle as mo
from paper_2605_05219_amd import feed_forward as FF

HALF = 2.0 ** -8


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def half_step(v, e):
    return e + HALF * (np.abs(v) + e) + 2.0 ** -134


def within(got, ref, bound):
    worst = np.abs(f64(got) - ref) - bound
    assert not np.isnan(worst).any() and worst.max() <= 0, float(worst.max())


def checked_step(ff, y, stream, k=0):
    """One step, checked; returns what it returned."""
    import torch
    before, w = f64(stream), {name: f64(t) for name, t in ff.w.items()}
    (s, es), (x, ex) = bo.block_norm(f64(y), None, None, None, before, w["norm"], None, "none", "rms", eps_pre=1e-6)
    out = ff.step(y, stream)
    torch.cuda.synchronize()
    T = stream.shape[0]
    held = {name: t[:T] for name, t in ff.held.items()}
    within(held["x"], x, half_step(x, ex))
    x = f64(held["x"])
    if "router" not in w:
        assert out is None
        h, eh = lo.linear_act(x, w["gate"], None, "silu", w["up"])
        within(held["h"], h, half_step(h, eh))
        o, eo = lo.linear_act(f64(held["h"]), w["down"], None, residual=s)
        within(stream, o, eo + es)
        return out
    within(stream, s, es)
    add, eadd = None, 0.0
    if "shared_gate" in w:
        h, eh = lo.linear_act(x, w["shared_gate"], None, "silu", w["shared_up"])
        within(held["h"], h, half_step(h, eh))
        add, eadd = lo.linear_act(f64(held["h"]), w["shared_down"], None)
        eadd = half_step(add, eadd)
    _, _, (o, eo) = mo.moe(x, w["router"], None, w["gate_up"], w["down"], add, k)
    assert out.data_ptr() == held["out"].data_ptr() and out.shape == stream.shape
    within(out, o, half_step(o, eo + eadd))
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 40, 300])
def test_dense_blocks(T):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    stream = torch.randn(T, 256, generator=gen, device="cuda") * 2
    out = torch.randn(T, 256, generator=gen, device="cuda").bfloat16()
    for inner in (192, 640):
        out = checked_step(FF.FeedForward(FF.random_weights(256, inner, generator=gen)), out, stream)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 6, 70])
@pytest.mark.parametrize("shared", [0, 128])
def test_experts_between_dense_blocks(T, shared):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(10 * T + shared)
    stream = torch.randn(T, 128, generator=gen, device="cuda") * 2
    out = torch.randn(T, 128, generator=gen, device="cuda").bfloat16()
    for experts in (0, 12, 200, 0):
        ff = FF.FeedForward(FF.random_weights(128, 64, experts, shared if experts else 0, gen), 3 if experts else 0)
        out = checked_step(ff, out, stream, 3)
    # a batch that grows and one that shrinks, in the same object
    ff = FF.FeedForward(FF.random_weights(128, 64, 12, shared, gen), 3)
    for n in (T, 2 * T + 3, T):
        checked_step(ff, torch.randn(n, 128, generator=gen, device="cuda").bfloat16(), torch.randn(n, 128, generator=gen, device="cuda"), 3)


@pytest.mark.gpu
@pytest.mark.parametrize("experts", [0, 16])
@pytest.mark.parametrize("T", [1, 50])
def test_a_captured_step(experts, T):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T)
    blocks = [FF.FeedForward(FF.random_weights(192, 128, experts, 64 if experts else 0, gen), 4) for _ in range(2)]
    y = torch.randn(T, 192, generator=gen, device="cuda").bfloat16()
    start = torch.randn(T, 192, generator=gen, device="cuda")
    stream = start.clone()

    def step():
        out = y
        for b in blocks:
            out = b.step(out, stream)
        return out

    out = step()                                                            # buffers are made outside the graph
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stream.copy_(start)
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        y.mul_(0.7).add_(0.1 * i)
        stream.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        got = stream.clone(), None if out is None else out.clone()
        stream.copy_(start)
        again = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], stream) and (again is None or torch.equal(got[1], again))


@pytest.mark.gpu
def test_the_command_runs(capsys):
    for more in ([], ["--experts", "8", "--experts-per-token", "2", "--shared", "64"]):
        FF.main(["--tokens", "3", "--layers", "2", "--width", "128", "--inner", "64", "--steps", "2"] + more)
        assert "us a block" in capsys.readouterr().out


@pytest.mark.gpu
def test_a_capture_that_would_need_new_buffers_is_refused():
    import torch
    ff = FF.FeedForward(FF.random_weights(128, 64))
    stream, y = torch.zeros(4, 128, device="cuda"), torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(graph):
            ff.step(y, stream)
    ff.step(y, stream)
    first = ff.held["x"]
    ff.step(y.repeat(9, 1), stream.repeat(9, 1))
    assert any(t is first for t in ff.outgrown)                              # a graph that has it may go on


@pytest.mark.gpu
@pytest.mark.parametrize("experts", [0, 8])
def test_a_step_of_no_tokens_and_one_without_a_block_before_it(experts):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    ff = FF.FeedForward(FF.random_weights(128, 64, experts, 64 if experts else 0, gen), 2)
    out = ff.step(torch.empty(0, 128, device="cuda", dtype=torch.bfloat16), torch.empty(0, 128, device="cuda"))
    assert out is None if not experts else out.shape == (0, 128)
    stream = torch.randn(5, 128, generator=gen, device="cuda")
    alone, added = stream.clone(), stream.clone()
    first = ff.step(None, alone)
    first = None if first is None else first.clone()
    second = ff.step(torch.zeros(5, 128, device="cuda", dtype=torch.bfloat16), added)
    torch.cuda.synchronize()
    assert torch.equal(alone, added) and (first is None or torch.equal(first, second))


@pytest.mark.gpu
def test_a_step_that_finds_no_buffers_leaves_the_stream_as_it_was():
    import torch
    from paper_2605_05219_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(3)
    stream, y = torch.randn(6, 128, generator=gen, device="cuda"), torch.randn(6, 128, generator=gen, device="cuda").bfloat16()
    want = stream.clone()
    with pytest.raises(B.GdnError):                                   # no experts for a token: no workspace has a size
        FF.FeedForward(FF.random_weights(128, 64, 8, generator=gen), 0).step(y, stream)
    torch.cuda.synchronize()
    assert torch.equal(stream, want)
