"""Oracle of the paged key/value cache's operators.  TEST INFRASTRUCTURE ONLY.

Plain numpy in fp64, each formula of include/attn_paged.h per request and head; it shares no code with the library.
Attention over a request's rows is attn_oracle's."""
from __future__ import annotations

import math

import numpy as np


def rope_freqs(rot, base=10000.0, kind="plain", factor=1.0, context=0.0, fast=32.0, slow=1.0):
    """(rot / 2 angles per position, amplitude)."""
    if kind == "base":
        base = base * factor ** (rot / (rot - 2.0))
    f = np.array([base ** (-2.0 * p / rot) for p in range(rot // 2)])
    if kind == "linear":
        return f / factor, 1.0
    if kind != "ramp":
        return f, 1.0
    pair = lambda turns: rot * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot - 1)
    out = []
    for p, x in enumerate(f):
        slowed = min(max((p - lo) / max(hi - lo, 0.001), 0.0), 1.0)
        out.append(x * (1 - slowed) + x / factor * slowed)
    return np.array(out), 0.1 * math.log(factor) + 1.0


def rotate(x, pos, freqs, layout, amplitude):
    """x [n][H][d], tokens at positions pos, pos + 1, ...: the first 2 * freqs.size elements turned in pairs."""
    y = np.array(x, dtype=np.float64)
    m = freqs.size
    for i in range(y.shape[0]):
        for p in range(m):
            a, b = (p, p + m) if layout == "half" else (2 * p, 2 * p + 1)
            phi = float(pos + i) * float(freqs[p])
            u, w = x[i, :, a].astype(np.float64), x[i, :, b].astype(np.float64)
            y[i, :, a] = amplitude * (u * math.cos(phi) - w * math.sin(phi))
            y[i, :, b] = amplitude * (w * math.cos(phi) + u * math.sin(phi))
    return y


def logits(q, k_all, start, scale):
    """[H_q][n][start + n] scaled logits, -inf where a token does not see the row."""
    q, k_all = np.asarray(q, np.float64), np.asarray(k_all, np.float64)
    n, H_q, _ = q.shape
    G = H_q // k_all.shape[1]
    x = np.stack([scale * q[:, h] @ k_all[:, h // G].T for h in range(H_q)])
    hidden = np.arange(k_all.shape[0])[None, :] > start + np.arange(n)[:, None]
    x[:, hidden] = -np.inf
    return x


def row_lse(q, k_all, start, scale):
    """[n][H_q]."""
    x = logits(q, k_all, start, scale)
    top = x.max(-1, keepdims=True)
    return (top[..., 0] + np.log(np.exp(x - top).sum(-1))).T


def key_weights(q, lse, k_all, start, scale, decay, w_in):
    """w_in [start][H_kv] or None; returns [start + n][H_kv]."""
    H_kv = k_all.shape[1]
    x = logits(q, k_all, start, scale)
    p = np.exp(x - np.asarray(lse, np.float64).T[:, :, None]).sum(1)          # [H_q][rows]
    w = p.reshape(H_kv, -1, k_all.shape[0]).sum(1).T
    if w_in is not None:
        w[:start] += decay * np.asarray(w_in, np.float64)
    return w


def rows_kept(w, keep, first, recent):
    """w [rows] of one head: the row numbers kept, ascending."""
    rows = len(w)
    keep = min(keep, rows)
    middle = range(first, rows - recent)
    value = lambda j: (1, 0.0) if math.isnan(w[j]) else (0, -float(w[j]))  # noqa: E731
    best = sorted(middle, key=lambda j: value(j) + (j,))[:keep - first - recent] if keep < rows else list(middle)
    return sorted(list(range(first)) + list(best) + list(range(rows - recent, rows)))
