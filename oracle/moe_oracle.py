"""Oracle of the mixture of experts.  TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product path, and it shares no
code with the HIP library.

The definition in fp64, token by token and choice by choice, with the three roundings that the definition has (the router's sum and the key to
fp32, p * act(gate) * up to bf16), and a bound on what fp32 arithmetic may be off by beside every value.

Pins (tests/test_moe.py): a hand-worked case, one expert against the plain gated block, order and ties, keys that are never chosen.
"""
from __future__ import annotations

import numpy as np

from . import linear_oracle as lo

U23 = 2.0 ** -23


def to_bf16(a):
    """Nearest bf16 (ties to even) of fp64 values, as fp64: exact, by scaling each value's 8 significant bits to whole numbers."""
    a = np.asarray(a, np.float64)
    m, e = np.frexp(a)
    return np.where(np.isfinite(a), np.ldexp(np.rint(np.ldexp(m, 8)), e - 8), a)


def route(x, w_router, choice_bias, k, score="softmax", normalise=True, routed_scale=1.0):
    """(ids [T][k], -1 where there is none; weights [T][k]; bound of the weights' error)."""
    with np.errstate(all="ignore"):
        l32 = (x @ w_router.T).astype(np.float32)
        s = l32.astype(np.float64)
        key = 1 / (1 + np.exp(-s)) if score == "sigmoid" else s
        if choice_bias is not None:
            key = key + choice_bias
        key = key.astype(np.float32)
        T, E = key.shape
        ids, p, ep = np.full((T, k), -1, np.int64), np.zeros((T, k)), np.zeros((T, k))
        for t in range(T):
            order = [e for e in range(E) if key[t, e] != -np.inf]
            order.sort(key=lambda e: (1, 0.0, e) if np.isnan(key[t, e]) else (0, -float(key[t, e]), e))
            got = order[:k]
            n = len(got)
            ids[t, :n] = got
            if not n:
                continue
            l = s[t, got]
            if score == "sigmoid":
                ls = -np.logaddexp(0, -l)    # (by its logarithm: divided by their sum, sigmoids below fp64's range still count)
                w = np.exp(ls - (ls.max() if normalise and ls.max() != -np.inf else 0))
            else:
                w = np.exp(l - s[t].max())
                w = w / np.exp(s[t] - s[t].max()).sum()
                if normalise:                # (divided by their sum next; from the chosen ones' own largest, nothing is lost to underflow)
                    w = np.exp(l - l.max())
            if normalise:
                w = w / w.sum() if w.sum() != 0 else 0 * w
            span = np.nanmax(np.abs(s[t] - s[t, got].max()), initial=0.0, where=np.isfinite(s[t])) + np.nanmax(np.abs(l), initial=0.0, where=np.isfinite(l))
            p[t, :n] = w * float(np.float32(routed_scale))
            ep[t, :n] = np.abs(p[t, :n]) * (2 * span + 64) * 2.0 ** -24 + 2.0 ** -126
    return ids, p, ep


def experts(x, ids, p, ep, w_gate_up, w_down, add, act):
    """(y [T][D], bound of fp32's error) for given choices; a choice of weight zero is left out."""
    T, D = x.shape
    F, K = w_down.shape[2], ids.shape[1]                  # (a sum may go over all choices at once)
    y = np.zeros((T, D)) if add is None else np.array(add, np.float64)
    e = np.zeros((T, D))
    size = np.abs(y)
    for ex in range(w_down.shape[0]):
        t, j = np.nonzero((ids == ex) & (p != 0))
        if not t.size:
            continue
        xe = x[t]
        gate, up = (lo.linear(xe, w_gate_up[ex][h]) for h in (slice(0, F), slice(F, 2 * F)))
        eg, eu = ((D + 8) * U23 * (np.abs(xe) @ np.abs(w_gate_up[ex][h]).T) for h in (slice(0, F), slice(F, 2 * F)))
        a, ea = lo.act_with_bound(act, gate, eg)
        w, ew = p[t, j][:, None], ep[t, j][:, None]
        g, eg = a * up, ea * np.abs(up) + np.abs(a) * eu + ea * eu + U23 * np.abs(a * up)
        h, eh = w * g, np.abs(w) * eg + ew * (np.abs(g) + eg) + U23 * np.abs(w * g)
        hr = to_bf16(h)
        er = np.maximum(np.abs(to_bf16(h + eh) - hr), np.abs(to_bf16(h - eh) - hr))       # a step where a boundary is within reach
        down = np.abs(w_down[ex])
        o = hr @ w_down[ex].T
        y[t] += o                                                                          # (a token takes an expert once)
        e[t] += er @ down.T + (K * F + 8) * U23 * ((np.abs(hr) + er) @ down.T)
        size[t] += np.abs(o)
    return y, e + 20 * U23 * size


def moe(x, w_router, choice_bias, w_gate_up, w_down, add, k, act="silu", score="softmax", normalise=True, routed_scale=1.0):
    """(ids, (weights, bound), (y, bound)) of fp64 arrays widened exactly from the bits that the GPU gets."""
    ids, p, ep = route(x, w_router, choice_bias, k, score, normalise, routed_scale)
    return ids, (p, ep), experts(x, ids, p, ep, w_gate_up, w_down, add, act)
