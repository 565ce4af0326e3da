"""The feed-forward half of a layer on its residual stream, dense or a mixture of experts.

    python -m paper_2605_05219_amd.feed_forward --tokens 64 --layers 4 --experts 128

`FeedForward.step` takes the mixer's output and the stream: the norm adds the one to the other and makes the block's input, the block's two products (or its
router and experts, on top of a shared expert where there is one) follow.  A dense block adds its output to the stream itself; that of a mixture of experts is
returned, for the next norm to add.  Everything is computed inside the library.  The command draws random weights and reports the time of a step."""
from __future__ import annotations

import argparse
import time

from . import block, linear, moe


class FeedForward:
    """weights: "norm" (fp32 [D]); dense: "gate", "up" [F][D], "down" [D][F]; experts: "router" [E][D], "gate_up" [E][2 F][D], "down" [E][D][F], a
    "choice_bias" (fp32 [E]) where there is one, and of a shared expert "shared_gate", "shared_up" [F_s][D], "shared_down" [D][F_s] (bf16)."""

    def __init__(self, weights, experts_per_token=0, act="silu", score="softmax", normalise=True, routed_scale=1.0, stream_dtype="f32", eps=1e-6):
        self.w, self.act = weights, act
        D = int(weights["norm"].numel())
        self.norm = block.make_block_shape(D, "none", "rms", "bf16", stream_dtype, "bf16", eps_pre=eps)
        self.experts = None
        if "router" in weights:
            E, _, F = weights["down"].shape
            router = "f32" if weights["router"].element_size() == 4 else "bf16"
            self.experts = moe.make_moe_shape(E, experts_per_token, D, F, act, score, normalise, routed_scale, router)
        self.held, self.outgrown = {}, []                # buffers by name; a step on another stream, or one at the same time, takes another object

    def _room(self, name, rows, make):
        """The object's buffer of that name with at least so many rows.  One that is outgrown is kept: a captured graph may go on using it."""
        import torch
        t = self.held.get(name)
        if t is None or t.shape[0] < rows:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a step of the largest batch comes before the capture of a graph: its buffers are not the graph's")
            if t is not None:
                self.outgrown.append(t)
            t = self.held[name] = make(rows + rows // 4)
        return t[:rows]

    def step(self, y, stream):
        """y: what the block before gave, bf16 [T][D], or None where the stream has it; stream: [T][D], changed in place.  Returns what is still to be
        added to the stream (in a buffer of this object's), or None."""
        import torch
        w, (T, D) = self.w, stream.shape
        like = w["down"]
        rows = lambda cols: lambda n: torch.empty(n, cols, dtype=like.dtype, device=like.device)  # noqa: E731
        # every buffer before the first launch: what fails here leaves the stream as it was
        x = self._room("x", T, rows(D))
        inner = w["gate"] if self.experts is None else w.get("shared_gate")
        h = self._room("h", T, rows(inner.shape[0])) if inner is not None else None
        if self.experts is not None:
            out = self._room("out", T, rows(D))
            ws = self._room("workspace", moe.gdn_moe_workspace_bytes(self.experts, T), lambda n: torch.empty(n, dtype=torch.uint8, device=like.device))
        block.gdn_block_norm(self.norm, y, None, None, None, stream, w["norm"], None, stream if y is not None else None, x)
        if self.experts is None:
            linear.gdn_linear_act(x, w["gate"], None, h, self.act, w["up"])
            linear.gdn_linear_act(h, w["down"], None, stream, residual=stream)
            return None
        add = None
        if h is not None:
            linear.gdn_linear_act(x, w["shared_gate"], None, h, self.act, w["shared_up"])
            linear.gdn_linear_act(h, w["shared_down"], None, out)
            add = out
        moe.gdn_moe(self.experts, x, w["router"], w.get("choice_bias"), w["gate_up"], w["down"], add, out, None, None, ws)
        return out


def random_weights(D, F, experts=0, shared=0, generator=None, device="cuda"):
    """Weights of the sizes above, of a scale that keeps the stream's."""
    import torch
    normal = lambda *n: torch.randn(*n, generator=generator, device=device)  # noqa: E731
    bf = lambda *n: (normal(*n) * n[-1] ** -0.5).bfloat16()  # noqa: E731
    w = {"norm": 1 + 0.1 * normal(D)}
    if not experts:
        return {**w, "gate": bf(F, D), "up": bf(F, D), "down": bf(D, F)}
    w.update(router=bf(experts, D), gate_up=bf(experts, 2 * F, D), down=bf(experts, D, F))
    if shared:
        w.update(shared_gate=bf(shared, D), shared_up=bf(shared, D), shared_down=bf(D, shared))
    return w


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--inner", type=int, default=768)
    ap.add_argument("--experts", type=int, default=0)
    ap.add_argument("--experts-per-token", type=int, default=8)
    ap.add_argument("--shared", type=int, default=0, help="inner width of a shared expert")
    ap.add_argument("--steps", type=int, default=50)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(0)
    layers = [FeedForward(random_weights(a.width, a.inner, a.experts, a.shared, gen), min(a.experts_per_token, a.experts)) for _ in range(a.layers)]
    stream = torch.randn(a.tokens, a.width, generator=gen, device="cuda")
    mixed = [torch.randn(a.tokens, a.width, generator=gen, device="cuda").bfloat16() for _ in layers]

    def step():
        for layer, y in zip(layers, mixed):
            out = layer.step(y, stream)
            if out is not None:
                stream.add_(out)                         # (a program's next mixer would take it through its own norm)

    step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.steps):
        step()
    torch.cuda.synchronize()
    kind = f"{a.experts} experts, {min(a.experts_per_token, a.experts)} a token" if a.experts else "dense"
    print(f"{a.layers} blocks of {a.width} x {a.inner}, {kind}, {a.tokens} tokens: {(time.perf_counter() - t0) / a.steps * 1e6 / a.layers:.1f} us a block")


if __name__ == "__main__":
    main()
