"""The operators of a layer between its token mixers, and what each is measured on.

  norm     gdn_block_norm: the residual stream with the norm behind the last block, its gate and scale, and the norm before the next
  linear   gdn_linear_act: a projection with bias, activation (gated or not), scale and residual in its epilogue
  moe      gdn_moe:        a mixture-of-experts layer: router, choice, the experts' gated products, their weighted sum

Where `own` is false, run() computes them in elementary torch operations in 32 bits (the router's sums and keys, which decide a
choice, in 64), rounded once at the end; where it is true, through the framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
ROUTED_SCALE = 1.5      # of the cases whose router scores by sigmoids


# ----------------------------------------------------------------------------- the cases
def _norm(T, D, post="none", pre="rms", gate="none", gate_act="none", dtype="bf16", stream="bf16", scale=1.0, offset=0.0, pad=0):
    return dict(kind="norm", T=T, D=D, post=post, pre=pre, gate=gate, gate_act=gate_act, dtype=dtype, stream=stream, scale=scale,
                offset=offset, pad=pad)


def _linear(T, N, K, act="none", gated=False, bias=False, residual="none", out="bf16", scale=1.0, pad=0):
    return dict(kind="linear", T=T, N=N, K=K, act=act, gated=gated, bias=bias, residual=residual, out=out, scale=scale, pad=pad)


def _moe(T, E, k, D, F, act="silu", score="softmax", normalise=True, bias=False, add=False, router="bf16"):
    return dict(kind="moe", T=T, E=E, k=k, D=D, F=F, act=act, score=score, normalise=normalise, bias=bias, add=add, router=router)


def listed():
    return [
        # one token of a single user: launches and host time are all there is
        dict(name="norm_token", **_norm(1, 2048)),
        # a decoding batch whose stream is held in 32 bits
        dict(name="norm_decode", **_norm(64, 2048, stream="f32", offset=1.0)),
        # ragged suffixes of a wide layer: norms on both sides of the block, with a gate of the block's own, out of wider buffers
        dict(name="norm_ragged", **_norm(1777, 5120, "layer", "layer", "element", "sigmoid", "bf16", "f32", 0.7, 0.0, 24)),
        # the prompt of the layer group of the benchmark, 8192 tokens; a learned scale for each channel of the block
        dict(name="norm_prompt", **_norm(8192, 2048, "rms", "rms", "channel")),
        # the gate and up projections of one token: two weight matrices read once
        dict(name="linear_up_token", **_linear(1, 6144, 2048, "silu", True)),
        # the down projection of a decoding batch, onto the stream
        dict(name="linear_down_decode", **_linear(48, 2048, 6144, residual="bf16")),
        # ragged suffixes through a layer with biases, odd widths, 32-bit outputs
        dict(name="linear_ragged", **_linear(1401, 1733, 1600, "gelu", False, True, "f32", "f32", 0.5, 8)),
        # the gate and up projections of the prompt
        dict(name="linear_up_prompt", **_linear(8192, 6144, 2048, "silu", True)),
        # one token through eight of 128 experts
        dict(name="moe_token", **_moe(1, 128, 8, 2048, 768)),
        # a decoding batch that reaches nearly every expert
        dict(name="moe_decode", **_moe(64, 128, 8, 2048, 768)),
        # a short suffix over many small experts, balanced by a bias on the choice, on top of a shared expert's output
        dict(name="moe_many_experts", **_moe(200, 512, 10, 2048, 512, "silu", "sigmoid", True, True, True, "f32")),
        # a chunk of a prompt: some two hundred tokens an expert
        dict(name="moe_chunk", **_moe(2048, 64, 6, 2048, 1408, "gelu_tanh", "softmax", False)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        for key, v in _cost(c).items():
            most[c["kind"], key] = max(v, most.get((c["kind"], key), 0))
    while True:
        case = _draw_any(rng)
        if all(v <= most[case["kind"], key] for key, v in _cost(case).items()):
            return case


def _cost(case):
    w = dict(work(case))
    if case["kind"] == "moe":        # the plain form runs every token through every expert
        w["dense"] = case["T"] * case["E"] * case["D"] * case["F"]
    return w


def _draw_any(rng):
    kind = rng.choice(["norm", "linear", "linear", "moe", "moe"])
    if kind == "norm":
        post = rng.choice(["none", "rms", "layer"])
        return _norm(_log_int(rng, 1, 16384), 8 * _log_int(rng, 4, 1280), post, rng.choice(["rms", "rms", "layer", "none"]),
                     rng.choice(["none", "element", "token", "channel"]), rng.choice(["none", "sigmoid"]), rng.choice(["bf16", "bf16", "f32"]),
                     rng.choice(["bf16", "f32"]), rng.choice([1.0, 0.5]), rng.choice([0.0, 1.0]), 8 * rng.randrange(3))
    if kind == "linear":
        return _linear(_log_int(rng, 1, 8192), _log_int(rng, 16, 8192), 64 * _log_int(rng, 1, 128),
                       rng.choice(["none", "silu", "gelu", "gelu_tanh", "relu", "relu2", "sigmoid"]), rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice(["none", "bf16", "f32"]), rng.choice(["bf16", "f32"]), rng.choice([1.0, 0.25]), 8 * rng.randrange(3))
    E = rng.choice([8, 16, 60, 64, 128, 256, 512])
    return _moe(_log_int(rng, 1, 2048), E, rng.randrange(1, min(E, 10) + 1), 64 * _log_int(rng, 4, 64), 64 * _log_int(rng, 2, 32),
                rng.choice(["silu", "silu", "gelu_tanh", "relu"]), rng.choice(["softmax", "sigmoid"]), rng.random() < 0.7, rng.random() < 0.4,
                rng.random() < 0.4, rng.choice(["bf16", "f32"]))


def _size(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    T = case["T"]
    if case["kind"] == "norm":
        D, a, b = case["D"], _size(case["dtype"]), _size(case["stream"])
        gate = {"none": 0, "element": T * D * a, "token": T * a, "channel": D * 4}[case["gate"]]
        params = 4 * D * ({"none": 0, "rms": 1, "layer": 2}[case["post"]] + {"none": 0, "rms": 1, "layer": 2}[case["pre"]])
        return {"bytes": T * D * (a + 2 * b + 2 * (case["pre"] != "none")) + gate + params, "flops": T * D * 12}
    if case["kind"] == "linear":
        N, K, two = case["N"], case["K"], 1 + case["gated"]
        residual = 0 if case["residual"] == "none" else T * N * _size(case["residual"])
        return {"bytes": T * K * 2 + two * N * K * 2 + two * 4 * N * case["bias"] + residual + T * N * _size(case["out"]),
                "flops": 2 * T * N * K * two}
    E, k, D, F = case["E"], case["k"], case["D"], case["F"]
    reached = E * (1 - (1 - k / E) ** T)                 # experts that some token chooses, by an even choice
    return {"bytes": reached * 3 * D * F * 2 + E * D * _size(case["router"]) + T * D * (4 + 2 * case["add"]) + T * k * 8,
            "flops": 2 * T * E * D + 2 * T * k * 3 * D * F}


# ----------------------------------------------------------------------------- the program's state
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, s=1.0, mean=0.0, dtype="f32"):
        return (torch.randn(*shape, generator=gen, device=dev) * s + mean).to(_DTYPES[dtype])

    def rows(n, width, pad, **kw):                       # n rows of a wider buffer
        return normal(n, width + pad, **kw)[:, :width]

    def out(n, width, pad, dtype):
        return torch.zeros(n, -(-width // 8) * 8 + pad, device=dev, dtype=_DTYPES[dtype])[:, :width]

    T, s = case["T"], dict(case=case)
    if case["kind"] == "norm":
        D, pad = case["D"], case["pad"]
        s["y"] = rows(T, D, pad, s=2.0, mean=0.3, dtype=case["dtype"])
        s["residual"] = rows(T, D, pad, s=4.0, mean=-0.2, dtype=case["stream"])
        s["gate"] = {"none": lambda: None, "element": lambda: rows(T, D, pad, dtype=case["dtype"]),
                     "token": lambda: normal(T, dtype=case["dtype"]), "channel": lambda: normal(D, s=0.3, mean=0.5)}[case["gate"]]()
        for side in ("post", "pre"):
            s["w_" + side] = normal(D, s=0.2, mean=1.0 - case["offset"]) if case[side] != "none" else None
            s["b_" + side] = normal(D, s=0.2) if case[side] == "layer" else None
        s["stream"] = out(T, D, pad, case["stream"])
        s["x"] = out(T, D, pad, "bf16") if case["pre"] != "none" else None
        if own:
            from paper_2605_05219_amd import block
            s["shape"] = block.make_block_shape(D, case["post"], case["pre"], case["dtype"], case["stream"], "bf16", case["gate"],
                                                case["gate_act"], EPS, EPS, case["scale"], case["offset"])
    elif case["kind"] == "linear":
        N, K, pad = case["N"], case["K"], case["pad"]
        s["x"] = rows(T, K, pad, dtype="bf16")
        s["w"] = normal(N, K, s=K ** -0.5, dtype="bf16")
        s["w_up"] = normal(N, K, s=K ** -0.5, dtype="bf16") if case["gated"] else None
        s["bias"] = normal(N, s=0.5) if case["bias"] else None
        s["bias_up"] = normal(N, s=0.5) if case["bias"] and case["gated"] else None
        s["residual"] = None
        if case["residual"] != "none":
            s["residual"] = rows(T, N, -N % 8 + pad, dtype=case["residual"])
        s["out"] = out(T, N, pad, case["out"])
    else:
        E, k, D, F = case["E"], case["k"], case["D"], case["F"]
        s["x"] = normal(T, D, dtype="bf16")
        s["w_router"] = normal(E, D, s=1.5 * D ** -0.5, dtype=case["router"])
        s["bias"] = normal(E, s=0.1) if case["bias"] else None
        s["w_gate_up"] = normal(E, 2 * F, D, s=D ** -0.5, dtype="bf16")
        s["w_down"] = normal(E, D, F, s=F ** -0.5, dtype="bf16")
        s["add"] = normal(T, D, dtype="bf16") if case["add"] else None
        s["out"] = torch.zeros(T, D, dtype=torch.bfloat16, device=dev)
        s["ids"] = torch.zeros(T, k, dtype=torch.int32, device=dev)
        s["weights"] = torch.zeros(T, k, device=dev)
        s["routed_scale"] = ROUTED_SCALE if case["score"] == "sigmoid" else 1.0
        if own:
            from paper_2605_05219_amd import moe
            s["shape"] = moe.make_moe_shape(E, k, D, F, case["act"], case["score"], case["normalise"], s["routed_scale"], case["router"])
            s["workspace"] = torch.empty(moe.gdn_moe_workspace_bytes(s["shape"], T), dtype=torch.uint8, device=dev)
    return s


# ----------------------------------------------------------------------------- the plain forms
def _act(name, z):
    if name == "silu":
        return z / (1 + (-z).exp())
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "relu":
        return z.clamp_min(0)
    if name == "relu2":
        return z.clamp_min(0) * z.clamp_min(0)
    if name == "sigmoid":
        return 1 / (1 + (-z).exp())
    return z


def _plain_norm(s):
    c = s["case"]

    def normed(v, kind, w, b):
        if kind == "layer":
            v = v - v.mean(-1, keepdim=True)
        v = v * ((v * v).mean(-1, keepdim=True) + EPS).rsqrt() * (w + c["offset"])
        return v if b is None else v + b

    y = s["y"].float()
    if c["post"] != "none":
        y = normed(y, c["post"], s["w_post"], s["b_post"])
    if s["gate"] is not None:
        g = s["gate"].float()
        if c["gate_act"] == "sigmoid":
            g = 1 / (1 + (-g).exp())
        y = y * (g[:, None] if c["gate"] == "token" else g)
    stream = s["residual"].float() + c["scale"] * y
    s["stream"].copy_(stream)
    if s["x"] is not None:
        s["x"].copy_(normed(stream, c["pre"], s["w_pre"], s["b_pre"]))
    return {"stream": s["stream"], "x": s["x"]}


def _plain_linear(s):
    c, x = s["case"], s["x"].float()

    def product(w, bias):
        z = x @ w.float().T
        return z if bias is None else z + bias

    a = _act(c["act"], product(s["w"], s["bias"]))
    if s["w_up"] is not None:
        a = a * product(s["w_up"], s["bias_up"])
    a = a * c["scale"]
    if s["residual"] is not None:
        a = a + s["residual"].float()
    s["out"].copy_(a)
    return {"y": s["out"]}


def _plain_moe(s):
    c, x = s["case"], s["x"]
    logits = (x.double() @ s["w_router"].double().T).float()
    key = logits.double() if c["score"] == "softmax" else 1 / (1 + (-logits.double()).exp())
    if s["bias"] is not None:
        key = key + s["bias"].double()
    ids = key.float().sort(dim=-1, descending=True, stable=True).indices[:, :c["k"]]
    if c["score"] == "softmax":
        p = (logits - logits.amax(-1, keepdim=True)).exp()
        p = p / p.sum(-1, keepdim=True)
    else:
        p = 1 / (1 + (-logits).exp())
    p = p.gather(1, ids)
    if c["normalise"]:
        p = p / p.sum(-1, keepdim=True)
    p = p * s["routed_scale"]
    if ids.numel() <= c["E"]:        # fewer choices than experts: the weights of each choice
        at = ids.reshape(-1)
        rows = x.float().repeat_interleave(c["k"], 0)[..., None]                          # [T k][D][1]
        h = torch.matmul(s["w_gate_up"][at].float(), rows)
        h = _act(c["act"], h[:, :c["F"]]) * h[:, c["F"]:]
        y = (torch.matmul(s["w_down"][at].float(), h).view(c["T"], c["k"], -1) * p[..., None]).sum(1)
    else:                            # every token through every expert, those not chosen with a weight of zero
        dense = torch.zeros_like(logits).scatter_(1, ids, p)                               # [T][E]
        h = torch.matmul(x.float(), s["w_gate_up"].float().transpose(1, 2).contiguous())  # [E][T][2F]
        h = _act(c["act"], h[..., :c["F"]]) * h[..., c["F"]:] * dense.T[..., None]
        h = h.transpose(0, 1).reshape(c["T"], -1)                                         # [T][E F]
        y = h @ s["w_down"].float().transpose(1, 2).reshape(-1, c["D"])
    if s["add"] is not None:
        y = y + s["add"].float()
    s["out"].copy_(y)
    s["ids"].copy_(ids)
    s["weights"].copy_(p)
    return {"y": s["out"], "ids": s["ids"], "weights": s["weights"]}


# ----------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "moe": _plain_moe}[kind](s)
    if kind == "norm":
        from paper_2605_05219_amd import block
        block.gdn_block_norm(s["shape"], s["y"], s["gate"], s["w_post"], s["b_post"], s["residual"], s["w_pre"], s["b_pre"], s["stream"],
                             s["x"])
        return {"stream": s["stream"], "x": s["x"]}
    if kind == "linear":
        from paper_2605_05219_amd import linear
        linear.gdn_linear_act(s["x"], s["w"], s["bias"], s["out"], s["case"]["act"], s["w_up"], s["bias_up"], s["residual"],
                              s["case"]["scale"])
        return {"y": s["out"]}
    from paper_2605_05219_amd import moe
    moe.gdn_moe(s["shape"], s["x"], s["w_router"], s["bias"], s["w_gate_up"], s["w_down"], s["add"], s["out"], s["ids"], s["weights"],
                s["workspace"])
    return {"y": s["out"], "ids": s["ids"], "weights": s["weights"]}


# ----------------------------------------------------------------------------- the definition in 64 bits
_EXACT_ACTS = {"none": lambda z: z, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
               "gelu_tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh"), "relu2": lambda z: torch.relu(z).square(),
               "sigmoid": torch.sigmoid}


def exact(case, seed):
    s = prepare(case, seed)
    wide = {key: v.double() for key, v in s.items() if isinstance(v, torch.Tensor) and not key.startswith("w_") and key != "ids"}
    if case["kind"] == "norm":
        def normed(v, side):
            if case[side] == "none":
                return v
            centre = v.mean(1, keepdim=True) if case[side] == "layer" else torch.zeros_like(v[:, :1])
            spread = torch.sqrt((v - centre).pow(2).sum(1, keepdim=True) / case["D"] + EPS)
            n = (v - centre) / spread * (s["w_" + side].double() + case["offset"])
            return n + s["b_" + side].double() if case[side] == "layer" else n

        branch = normed(wide["y"], "post")
        if case["gate"] != "none":
            g = torch.sigmoid(wide["gate"]) if case["gate_act"] == "sigmoid" else wide["gate"]
            branch = branch * (g.unsqueeze(1) if case["gate"] == "token" else g)
        stream = wide["residual"] + case["scale"] * branch
        return {"stream": stream, "x": normed(stream, "pre") if case["pre"] != "none" else None}

    act = _EXACT_ACTS[case["act"]]
    if case["kind"] == "linear":
        parts = [torch.nn.functional.linear(wide["x"], s[w].double(), wide.get(b)) for w, b in (("w", "bias"), ("w_up", "bias_up")) if s[w] is not None]
        y = case["scale"] * act(parts[0]) * (parts[1] if case["gated"] else 1.0)
        return {"y": y + wide["residual"] if case["residual"] != "none" else y}

    T, E, k, F = case["T"], case["E"], case["k"], case["F"]
    l32 = torch.nn.functional.linear(wide["x"], s["w_router"].double()).float()
    score = l32.double() if case["score"] == "softmax" else torch.sigmoid(l32.double())
    key = (score + wide["bias"] if case["bias"] else score).float().cpu().numpy()
    chosen = torch.from_numpy((-key).argsort(axis=1, kind="stable")[:, :k].copy()).to(l32.device)
    p = (torch.softmax(l32.double(), 1) if case["score"] == "softmax" else score).gather(1, chosen)
    p = s["routed_scale"] * (p / p.sum(1, keepdim=True) if case["normalise"] else p)
    y = wide["add"].clone() if case["add"] else torch.zeros(T, case["D"], dtype=torch.float64, device=p.device)
    for e in range(E):
        t, j = (chosen == e).nonzero(as_tuple=True)
        if t.numel():
            z = wide["x"][t] @ s["w_gate_up"][e].double().T
            y.index_add_(0, t, p[t, j][:, None] * ((act(z[:, :F]) * z[:, F:]) @ s["w_down"][e].double().T))
    return {"y": y, "ids": None, "weights": p}
