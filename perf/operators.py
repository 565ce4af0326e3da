"""The operators of an attention layer that keeps its keys and values in pages, and what each is measured on.

  rope      attn_rope_append:   rotary positions of q and k, and the append of k and v to the pages
  attend    attn_paged_prefill: causal attention of a chunk of new tokens over the pages, and each row's log-sum-exp on request
  weights   attn_key_weights:   the attention weight every cached row gathers from the chunk
  evict     attn_evict:         the rows with the most weight, copied to fresh pages

Where `own` is false, run() computes them in elementary torch operations over padded batches, in 32 bits (angles in 64)
rounded once at the end; where it is true, through the framework's entry points.  A case fixes every size (lengths are
drawn from the case's own `lengths` number), the seed of prepare() only the values and the page ids.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

ROPE_BASE = 10000.0
SCALED = dict(factor=16.0, context=8192, fast=32.0, slow=1.0)      # of the cases with scaled positions
DECAY = 0.9                                                       # of the gathered weights, per call


# ----------------------------------------------------------------------------- the cases
def _rope(n_req, heads_q, heads_kv, d, rot, layout, lo, hi, pos, page=64, dtype="bf16", scaled=False, lengths=0):
    return dict(kind="rope", n_req=n_req, heads_q=heads_q, heads_kv=heads_kv, d=d, rot=rot, layout=layout, lo=lo, hi=hi,
                prefix_lo=0, prefix_hi=200, pos=pos, page=page, dtype=dtype, scaled=scaled, shared=0, lengths=lengths)


def _over_cache(kind, n_req, heads_q, heads_kv, d, lo, hi, prefix_lo, prefix_hi, page=64, shared=0, gate=False,
                lse=False, lengths=0):
    return dict(kind=kind, n_req=n_req, heads_q=heads_q, heads_kv=heads_kv, d=d, lo=lo, hi=hi, prefix_lo=prefix_lo,
                prefix_hi=prefix_hi, page=page, shared=shared, gate=gate, lse=lse, lengths=lengths)


def _evict(n_req, heads_kv, d, lo, hi, keep, page=64, lengths=0):
    return dict(kind="evict", n_req=n_req, heads_q=heads_kv, heads_kv=heads_kv, d=d, lo=0, hi=0, prefix_lo=lo, prefix_hi=hi, keep=keep,
                page=page, shared=0, lengths=lengths)


def listed():
    return [
        # one token of a single user: launches and host time are all there is
        dict(name="rope_one_token", **_rope(1, 16, 2, 128, 128, "half", 1, 1, 5000)),
        # the prompt of the layer group of the benchmark, 8192 tokens
        dict(name="rope_prompt", **_rope(1, 16, 2, 128, 128, "half", 8192, 8192, 0)),
        # ragged suffixes far into long documents: a quarter of a wide head, interleaved pairs, scaled positions, projections in fp32
        dict(name="rope_far_batch", **_rope(16, 16, 4, 256, 64, "interleaved", 200, 1000, 900000, 32, "f32", True, 21)),
        # decoding of a full batch: one token per request behind 4 to 10 thousand rows
        dict(name="attend_decode", **_over_cache("attend", 64, 16, 2, 128, 1, 1, 4000, 10000, 64, lengths=22)),
        # one user deep in a long document: a single row over 150 thousand
        dict(name="attend_long", **_over_cache("attend", 1, 16, 2, 128, 1, 1, 150001, 150001, 128, lse=True)),
        # chunks of sixteen requests behind a few thousand rows, of which 2048 are a prefix that they share; gated outputs
        dict(name="attend_chunks", **_over_cache("attend", 16, 16, 2, 128, 200, 1000, 3000, 5000, 16, 2048, gate=True, lengths=23)),
        # the prompt: 8192 tokens over themselves; the weights that its rows gather are asked for next
        dict(name="attend_prompt", **_over_cache("attend", 1, 16, 2, 128, 8192, 8192, 0, 0, lse=True)),
        # the weights of a decoding batch
        dict(name="weights_decode", **_over_cache("weights", 64, 16, 2, 128, 1, 1, 4000, 10000, 64, lengths=22)),
        # the last chunk of a document: 500 tokens behind 7700 rows, one key/value head for every 4 query heads
        dict(name="weights_chunk", **_over_cache("weights", 1, 16, 4, 64, 500, 500, 7700, 7700, 32)),
        # the prompt
        dict(name="weights_prompt", **_over_cache("weights", 1, 16, 2, 128, 8192, 8192, 0, 0)),
        # one request back to a budget of 2000 rows
        dict(name="evict_one", **_evict(1, 2, 128, 8200, 8200, 2000)),
        # a batch of long requests, down to 8000 rows each
        dict(name="evict_batch", **_evict(32, 4, 128, 10000, 30000, 8000, 128, 24)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {c["name"]: work(c) for c in listed()}
    bytes_most, flops_most = max(w["bytes"] for w in most.values()), max(w["flops"] for w in most.values())
    while True:
        case = _draw_any(rng)
        w, lens, prefix = work(case), *_lengths(case)
        padded = case["n_req"] * case["heads_q"] * max(lens) * max(p + n for p, n in zip(prefix, lens))
        if w["bytes"] <= bytes_most and w["flops"] <= flops_most and padded <= 16 * 8192 * 8192:
            return case


def _draw_any(rng):
    kind = rng.choice(["rope", "attend", "attend", "attend", "weights", "weights", "evict"])
    lengths = rng.randrange(1 << 30)
    page = rng.choice([16, 32, 64, 128, 256])
    d = rng.choice([64, 128, 128, 256])
    heads = rng.choice([(16, 2), (16, 4), (32, 4), (8, 8), (6, 2), (8, 1)])
    if kind == "rope":
        lo = _log_int(rng, 1, 4000)
        return _rope(_log_int(rng, 1, 64), *heads, d, 16 * rng.randrange(1, d // 16 + 1), rng.choice(["half", "interleaved"]), lo,
                     min(2 * lo, 8192), rng.choice([0, _log_int(rng, 1, 2000000)]), page, rng.choice(["bf16", "bf16", "f32"]),
                     rng.random() < 0.4, lengths)
    if kind == "evict":
        lo = _log_int(rng, 100, 40000)
        return _evict(_log_int(rng, 1, 32), heads[1], d, lo, 2 * lo, _log_int(rng, 16, 2 * lo), page, lengths)
    prefix = _log_int(rng, 1, 10000)
    if rng.random() < 0.4:           # decoding, or a few tokens at once
        few = rng.choice([1, 1, 1, 4])
        if rng.random() < 0.25:      # behind a long cache
            prefix = _log_int(rng, 10000, 150000)
        lo, hi, n_req = 1, few, _log_int(rng, 1, 96)
    else:
        lo = _log_int(rng, 2, 4000)
        hi, n_req = min(2 * lo, 8192), _log_int(rng, 1, 32)
    shared = 256 * rng.randrange(1, 9) if kind == "attend" and prefix > 2560 and rng.random() < 0.3 else 0
    return _over_cache(kind, n_req, *heads, d, lo, hi, prefix, 2 * prefix if prefix <= 20000 else prefix, page, shared,
                       kind == "attend" and rng.random() < 0.3, kind == "attend" and rng.random() < 0.5, lengths)


def _lengths(case):
    """(new tokens, rows held before) of every request."""
    rng = np.random.default_rng(case["lengths"])
    lens = rng.integers(case["lo"], case["hi"] + 1, case["n_req"])
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, case["n_req"])
    return [int(x) for x in lens], [int(x) for x in prefix]


def _kept(case):
    """(first rows kept, last rows kept, rows kept in all) of every request."""
    lens, prefix = _lengths(case)
    keep = [min(case["keep"], n) for n in prefix]
    return [min(4, m) for m in keep], [min(64, m // 2) if m > 8 else 0 for m in keep], keep


def work(case):
    lens, prefix = _lengths(case)
    H, K, d = case["heads_q"], case["heads_kv"], case["d"]
    T, rows = sum(lens), sum(prefix) + sum(lens)
    pairs = sum(n * c + n * (n + 1) // 2 for n, c in zip(lens, prefix))      # (token, visible row)
    if case["kind"] == "rope":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": T * d * (H + 2 * K) * (size + 2), "flops": T * (H + K) * (case["rot"] // 2) * 6}
    if case["kind"] == "attend":
        distinct = rows - (case["n_req"] - 1) * min(case["shared"], min(prefix))
        return {"bytes": T * H * d * (4 + 2 * case["gate"]) + 4 * T * H * case["lse"] + distinct * K * d * 4, "flops": pairs * H * d * 4}
    if case["kind"] == "weights":
        return {"bytes": T * H * (2 * d + 4) + rows * K * (2 * d + 8), "flops": pairs * H * d * 2}
    kept = sum(_kept(case)[2])
    return {"bytes": rows * K * 4 + kept * K * (8 * d + 4 + 4 + 4), "flops": rows * K}


# ----------------------------------------------------------------------------- the program's state
def _freqs(rot, scaled):
    """Radians per position of each pair, and the factor on cosine and sine.  Scaled: a pair that turns more than `fast`
    times in the trained context keeps its frequency, one that turns less than `slow` times is slowed by `factor`, those
    between by a ramp over the pair's index; the factor is 0.1 ln(factor) + 1."""
    p = np.arange(rot // 2, dtype=np.float64)
    f = ROPE_BASE ** (-2.0 * p / rot)
    if not scaled:
        return f, 1.0
    at = lambda turns: rot * math.log(SCALED["context"] / (turns * 2 * math.pi)) / (2 * math.log(ROPE_BASE))  # noqa: E731
    lo, hi = max(math.floor(at(SCALED["fast"])), 0), min(math.ceil(at(SCALED["slow"])), rot - 1)
    slow = np.clip((p - lo) / max(hi - lo, 0.001), 0.0, 1.0)
    return f * (1 - slow) + f / SCALED["factor"] * slow, 0.1 * math.log(SCALED["factor"]) + 1.0


def prepare(case, seed):
    dev = torch.device("cuda")
    gen, rng = torch.Generator(device=dev).manual_seed(seed), np.random.default_rng(seed)
    normal = lambda *shape, s=1.0: torch.randn(*shape, generator=gen, device=dev) * s  # noqa: E731
    H, K, d, P, R = case["heads_q"], case["heads_kv"], case["d"], case["page"], case["n_req"]
    lens, prefix = _lengths(case)
    T, total = sum(lens), [c + n for c, n in zip(prefix, lens)]
    s = dict(case=case, H=H, K=K, d=d, P=P, R=R, T=T, n_max=max(lens), L_max=max(total), rows=sum(total), scale=d ** -0.5)

    # every request's pages, whole ones of a shared prefix once; ids in no order
    shared = min(case["shared"], min(prefix)) // P
    pages = [-(-n // P) for n in total]
    fresh = [n - shared for n in pages]
    new = [0] * R
    if case["kind"] == "evict":
        first, recent, keep = _kept(case)
        new = [-(-m // P) for m in keep]
    ids = rng.permutation(shared + sum(fresh) + sum(new)).astype(np.int32)
    own_cu = shared + np.concatenate([[0], np.cumsum(fresh)])
    listed_ids = [np.concatenate([ids[:shared], ids[own_cu[r]:own_cu[r + 1]]]) for r in range(R)]
    s["page_cu"] = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    s["page_ids"] = np.concatenate(listed_ids).astype(np.int32)
    s["cu"] = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    s["start"] = np.asarray(prefix, np.int32)

    on = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int64)).to(dev)  # noqa: E731
    table = np.zeros((R, max(pages)), np.int64)
    for r in range(R):
        table[r, :pages[r]] = listed_ids[r]
    s.update(d_table=on(table), d_cu=on(s["cu"]), d_len=on(lens), d_start=on(s["start"]), d_total=on(total),
             d_total_cu=on(np.concatenate([[0], np.cumsum(total)])))

    if case["kind"] == "weights":
        s["k_pool"] = normal(ids.size, K, P, d).bfloat16()
    else:
        s["k_pool"] = normal(ids.size, K, P, d).bfloat16()
        s["v_pool"] = normal(ids.size, K, P, d).half()
    if case["kind"] == "rope":
        made = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["q"], s["k"], s["v"] = (normal(T, h, d).to(made) for h in (H, K, K))
        s["freqs"], s["amplitude"] = _freqs(case["rot"], case["scaled"])
        s["pos"] = (case["pos"] + rng.integers(0, 100, R)).astype(np.int32) if case["pos"] else np.zeros(R, np.int32)
        s["d_freqs"], s["d_pos"] = torch.from_numpy(s["freqs"]).to(dev), on(s["pos"])
        s["q_out"] = torch.zeros(T, H, d, dtype=torch.bfloat16, device=dev)
    elif case["kind"] == "evict":
        s["w_pool"] = torch.exp(normal(ids.size, K, P, s=2.0))
        s["first"], s["recent"], s["keep"] = (np.asarray(x, np.int32) for x in (first, recent, keep))
        s["total"] = np.asarray(total, np.int32)
        s["new_cu"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        s["new_ids"] = ids[shared + sum(fresh):]
        new_table = np.zeros((R, max(new)), np.int64)
        for r in range(R):
            new_table[r, :new[r]] = s["new_ids"][s["new_cu"][r]:s["new_cu"][r + 1]]
        s.update(d_new_table=on(new_table), d_first=on(first), d_recent=on(recent), d_keep=on(keep),
                 d_keep_cu=on(np.concatenate([[0], np.cumsum(keep)])), kept=sum(keep), keep_max=max(keep))
        s["index"] = torch.zeros(sum(keep) * K, dtype=torch.int32, device=dev)
    else:
        s["q"] = normal(T, H, d, s=2.0).bfloat16()
        if case["kind"] == "attend":
            s["gate"] = normal(T, H, d).bfloat16() if case["gate"] else None
            s["o"] = torch.zeros(T, H, d, dtype=torch.bfloat16, device=dev)
            s["lse"] = torch.zeros(T, H, device=dev) if case["lse"] else None
        else:
            s["lse"] = _plain_logits(s)[1]
            s["w_in"] = torch.exp(normal(ids.size, K, P))
            s["w_out"] = torch.zeros(ids.size, K, P, device=dev)
    if own:
        from paper_2605_05219_amd import attention, paged
        s["shape"] = attention.make_attn_shape(H, K, d, "bf16")
        if case["kind"] == "rope":
            s["rope"] = paged.make_attn_rope(s["freqs"], case["layout"], s["amplitude"], case["dtype"])
        n_rows = int(s["rows"]) if case["kind"] == "evict" else T
        s["workspace"] = torch.empty(paged.attn_paged_workspace_bytes(s["shape"], R, n_rows, s["page_ids"].size + sum(new)),
                                     dtype=torch.uint8, device=dev)
    return s


# ----------------------------------------------------------------------------- the plain forms
def _each(s, lens, cu, count):
    """(request, index inside it) of `count` ragged entries."""
    req = torch.repeat_interleave(torch.arange(s["R"], device=lens.device), lens, output_size=count)
    return req, torch.arange(count, device=lens.device) - cu[req]


def _plain_rope(s):
    c = s["case"]
    req, i = _each(s, s["d_len"], s["d_cu"], s["T"])
    phi = (s["d_pos"][req] + i).double()[:, None] * s["d_freqs"]                     # [T][rot / 2]
    cos, sin = (phi.cos() * s["amplitude"])[:, None], (phi.sin() * s["amplitude"])[:, None]

    def rotate(x):
        half, y = c["rot"] // 2, x.double().clone()
        a, b = (slice(0, half), slice(half, c["rot"])) if c["layout"] == "half" else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
        u, w = x[..., a].double(), x[..., b].double()
        y[..., a] = u * cos - w * sin
        y[..., b] = w * cos + u * sin
        return y.bfloat16()

    row = s["d_start"][req] + i
    page = s["d_table"][req, row // s["P"]]
    s["q_out"].copy_(rotate(s["q"]))
    s["k_pool"][page, :, row % s["P"]] = rotate(s["k"])
    s["v_pool"][page, :, row % s["P"]] = s["v"].half()
    return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _rows_of(s, pool):
    """A pool's rows as a padded batch in 32 bits: [R][K][L_max][...]."""
    j = torch.arange(s["L_max"], device=pool.device)
    return pool[s["d_table"][:, j // s["P"]], :, j % s["P"]].float().transpose(1, 2)


def _plain_logits(s):
    """Padded logits [R][K][n_max * G][L_max] with -inf where nothing is seen, and the log-sum-exp [T][H] of the tokens' rows."""
    R, K, H, d = s["R"], s["K"], s["H"], s["d"]
    G, n, L = H // K, s["n_max"], s["L_max"]
    req, i = _each(s, s["d_len"], s["d_cu"], s["T"])
    q = torch.zeros(R, n, H, d, device=s["q"].device)
    q[req, i] = s["q"].float()
    q = q.view(R, n, K, G, d).transpose(1, 2).reshape(R, K, n * G, d)
    logits = torch.matmul(q, _rows_of(s, s["k_pool"]).transpose(2, 3)).mul_(s["scale"]).view(R, K, n, G, L)
    t, j = torch.arange(n, device=q.device), torch.arange(L, device=q.device)
    seen = (j <= s["d_start"][:, None, None] + t[:, None]) & (t[:, None] < s["d_len"][:, None, None])      # [R][n][L]
    logits.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = logits.amax(-1).clamp_min(-1e30)
    total = torch.zeros_like(top)
    total += (logits - top[..., None]).exp_().sum(-1)
    lse = (top + total.log()).transpose(1, 2).reshape(R, n, H)
    return logits, lse[req, i].contiguous()


def _plain_attend(s):
    R, K, H, d, n = s["R"], s["K"], s["H"], s["d"], s["n_max"]
    logits, lse = _plain_logits(s)
    top = logits.amax(-1, keepdim=True).clamp_min(-1e30)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True).clamp_min(1e-30)
    v = _rows_of(s, s["v_pool"])
    v = v * (torch.arange(s["L_max"], device=v.device) < s["d_total"][:, None])[:, None, :, None]
    o = torch.matmul(p.view(R, K, -1, s["L_max"]), v).view(R, K, n, H // K, d) / total
    req, i = _each(s, s["d_len"], s["d_cu"], s["T"])
    o = o.transpose(1, 2).reshape(R, n, H, d)[req, i]
    if s["gate"] is not None:
        o = o / (1.0 + (-s["gate"].float()).exp())
    s["o"].copy_(o.bfloat16())
    if s["lse"] is not None:
        s["lse"].copy_(lse)
    return {"o": s["o"], "lse": s["lse"]}


def _plain_weights(s):
    R, K, H, n = s["R"], s["K"], s["H"], s["n_max"]
    logits, _ = _plain_logits(s)
    req, i = _each(s, s["d_len"], s["d_cu"], s["T"])
    lse = torch.zeros(R, n, H, device=logits.device)
    lse[req, i] = s["lse"]
    p = logits.sub_(lse.view(R, n, K, H // K).transpose(1, 2)[..., None]).exp_()
    gathered = p.sum((2, 3))                                                        # [R][K][L_max]
    req, j = _each(s, s["d_total"], s["d_total_cu"], s["rows"])
    page, row = s["d_table"][req, j // s["P"]], j % s["P"]
    held = (j < s["d_start"][req])[:, None]
    s["w_out"][page, :, row] = torch.where(held, s["w_in"][page, :, row] * DECAY, torch.zeros((), device=page.device)) + gathered[req, :, j]
    return {"w": s["w_out"]}


def _plain_evict(s):
    R, K, P, L = s["R"], s["K"], s["P"], s["L_max"]
    dev = s["k_pool"].device
    j = torch.arange(L, device=dev)
    total = s["d_total"][:, None]
    always = (j < s["d_first"][:, None]) | (j >= total - s["d_recent"][:, None])
    w = _rows_of(s, s["w_pool"])                                                    # [R][K][L]
    w = torch.where((j >= total)[:, None], float("-inf"), torch.where(always[:, None], float("inf"), w))
    order = w.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros(R, K, L, dtype=torch.bool, device=dev)
    kept.scatter_(2, order, (j < s["d_keep"][:, None])[:, None].expand(R, K, L).contiguous())
    at = torch.where(kept, kept.cumsum(-1) - 1, s["keep_max"])                      # the rows left out go behind the last place
    rows = torch.zeros(R, K, s["keep_max"] + 1, dtype=torch.int64, device=dev).scatter_(2, at, j.expand(R, K, L).contiguous())
    req, i = _each(s, s["d_keep"], s["d_keep_cu"], s["kept"])
    g = torch.arange(K, device=dev)
    src = rows[req, :, i]                                                           # [kept][K]
    s["index"][K * s["d_keep_cu"][req][:, None] + g * s["d_keep"][req][:, None] + i[:, None]] = src.int()
    page, row = s["d_table"][req[:, None], src // P], src % P
    to_page, to_row = s["d_new_table"][req, i // P], i % P
    out = {"index": s["index"]}
    for name in ("k_pool", "v_pool", "w_pool"):
        s[name][to_page, :, to_row] = s[name][page, g, row]
        out[name] = s[name]
    return out


# ----------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"rope": _plain_rope, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}[kind](s)
    from paper_2605_05219_amd import paged
    if kind == "rope":
        paged.attn_rope_append(s["shape"], s["rope"], s["q"], s["k"], s["v"], s["cu"], s["pos"], s["start"], s["k_pool"], s["v_pool"],
                               s["page_cu"], s["page_ids"], s["q_out"], s["workspace"])
        return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if kind == "attend":
        paged.attn_paged_prefill(s["shape"], s["q"], s["gate"], s["cu"], s["start"], s["k_pool"], s["v_pool"], s["page_cu"], s["page_ids"],
                                 s["o"], s["lse"], s["workspace"])
        return {"o": s["o"], "lse": s["lse"]}
    if kind == "weights":
        paged.attn_key_weights(s["shape"], s["q"], s["lse"], s["cu"], s["start"], s["k_pool"], s["page_cu"], s["page_ids"], DECAY,
                               s["w_in"], s["w_out"], s["workspace"])
        return {"w": s["w_out"]}
    paged.attn_evict(s["shape"], s["total"], s["keep"], s["first"], s["recent"], s["k_pool"], s["v_pool"], s["w_pool"], s["page_cu"],
                     s["page_ids"], s["new_cu"], s["new_ids"], s["index"], s["workspace"])
    return {"index": s["index"], "k_pool": s["k_pool"], "v_pool": s["v_pool"], "w_pool": s["w_pool"]}


# ----------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    lens, prefix = _lengths(case)
    H, K, d, P = s["H"], s["K"], s["d"], s["P"]
    G, cu, dev = H // K, s["cu"], s["k_pool"].device

    def places(r, count, cu=s["page_cu"], ids=s["page_ids"]):
        j = np.arange(count)
        return torch.from_numpy(ids[cu[r] + j // P].astype(np.int64)).to(dev), torch.from_numpy(j % P).to(dev)

    if case["kind"] == "rope":
        q, k_pool, v_pool = s["q"].double(), s["k_pool"].double(), s["v_pool"].double()
        k, v = s["k"].double(), s["v"].double()
        for r, (n, c) in enumerate(zip(lens, prefix)):
            angle = torch.outer(torch.arange(n, dtype=torch.float64) + int(s["pos"][r]), torch.from_numpy(s["freqs"]))
            turn = torch.polar(torch.full_like(angle, s["amplitude"]), angle).to(dev)[:, None]
            for x in (q, k):
                part = x[cu[r]:cu[r + 1], :, :case["rot"]]
                pairs = part.unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (-1, 2))
                turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
                x[cu[r]:cu[r + 1], :, :case["rot"]] = (turned.transpose(-1, -2) if case["layout"] == "half" else turned).flatten(-2)
            page, row = places(r, c + n)
            k_pool[page[c:], :, row[c:]] = k[cu[r]:cu[r + 1]]
            v_pool[page[c:], :, row[c:]] = v[cu[r]:cu[r + 1]]
        return {"q": q, "k_pool": k_pool, "v_pool": v_pool}

    if case["kind"] == "evict":
        out = {x: s[x].double() for x in ("k_pool", "v_pool", "w_pool")}
        for r, n in enumerate(prefix):
            page, row = places(r, n)
            w = s["w_pool"][page, :, row].double().cpu().numpy()                       # [n][K]
            first, recent, keep = int(s["first"][r]), int(s["recent"][r]), int(s["keep"][r])
            for g in range(K):
                middle = np.arange(first, n - recent)
                best = middle[np.lexsort((middle, -w[middle, g]))][:keep - first - recent]
                rows = torch.from_numpy(np.sort(np.concatenate([np.arange(first), best, np.arange(n - recent, n)]))).to(dev)
                to_page, to_row = places(r, keep, s["new_cu"], s["new_ids"])
                for x in out:
                    out[x][to_page, g, to_row] = s[x][page[rows], g, row[rows]].double()
        return {"index": None, **out}

    o = torch.zeros(s["T"], H, d, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["T"], H, dtype=torch.float64, device=dev)
    w_out = s["w_out"].double() if case["kind"] == "weights" else None
    for r, (n, c) in enumerate(zip(lens, prefix)):
        page, row = places(r, c + n)
        hidden = torch.arange(c + n, device=dev)[None] > c + torch.arange(n, device=dev)[:, None]
        for g in range(K):
            k = s["k_pool"][page, g, row].double()
            gathered = torch.zeros(c + n, dtype=torch.float64, device=dev)
            for h in range(g * G, (g + 1) * G):
                x = (s["q"][cu[r]:cu[r + 1], h].double() @ k.T * d ** -0.5).masked_fill_(hidden, float("-inf"))
                if case["kind"] == "weights":
                    gathered += (x - s["lse"][cu[r]:cu[r + 1], h].double()[:, None]).exp_().sum(0)
                    continue
                z = torch.logsumexp(x, -1)
                lse[cu[r]:cu[r + 1], h] = z
                o[cu[r]:cu[r + 1], h] = (x - z[:, None]).exp_() @ s["v_pool"][page, g, row].double()
            if case["kind"] == "weights":
                gathered[:c] += DECAY * s["w_in"][page[:c], g, row[:c]].double()
                w_out[page, g, row] = gathered
    if case["kind"] == "weights":
        return {"w": w_out}
    if s["gate"] is not None:
        o = o * torch.sigmoid(s["gate"].double())
    return {"o": o, "lse": lse if case["lse"] else None}
