"""Oracle of the residual stream between two blocks of a layer.  TEST INFRASTRUCTURE ONLY: imported by the tests, never by the
product path, and it shares no code with the HIP library.

The definition in fp64, row by row, with a bound on what fp32 arithmetic may be off by beside every value:
    s[t] = r[t] + scale * g[t] * N_post(y[t]),   x[t] = N_pre(s[t]),
    N(v) = (v - m) / sqrt(mean((v - m)^2) + eps) * (w + offset) + b.

The bound, with u = 2^-24 (half a step of fp32): a sum of D terms is off by at most ADDS u sum|terms| (a thread adds at most 32,
six butterfly steps add the lanes, 16 waves' sums follow, and the products with 1/D round).  So the mean of v is off by ADDS u mean|v|, and the
deviations v - m by e = ev + mean(ev) + (ADDS + 1) u (|v| + mean|v|) for inputs that are off by ev.  The root mean square of a row that is off by e moves
by at most the root mean square of e; with the sum of squares' own ADDS u / 2, the root's and the quotient's u, the factor 1 / sqrt is off by
a relative rms(e) / sigma + (ADDS / 2 + 4) u.  Products and the last sum round three times more.

Pins (tests/test_block.py): hand-worked rows, the moments of a normalised row, invariance under scale and shift.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
ADDS = 64


def normalise(v, ev, kind, w, b, offset, eps):
    """(N(v), bound) of fp64 rows [T][D] whose elements are off by at most ev."""
    if kind == "none":
        return v, ev
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    e = ev
    if kind == "layer":
        e = ev + ev.mean(1, keepdims=True) + (ADDS + 1) * U * (np.abs(v) + np.abs(v).mean(1, keepdims=True))
    c = v - mean
    sigma = np.sqrt((c * c).mean(1, keepdims=True) + eps)
    weight = w + offset
    n = c / sigma * weight
    bound = (e / sigma) * np.abs(weight) + np.abs(n) * (np.sqrt((e * e).mean(1, keepdims=True)) / sigma + (ADDS / 2 + 8) * U)
    # (the sum w + offset rounds; so does the last one with b)
    bound = bound * 1.001 + U * np.abs(n)
    if b is not None:
        n = n + b
        bound = bound + U * np.abs(n)
    return n, bound


def block_norm(y, gate, w_post, b_post, r, w_pre, b_pre, post, pre, gate_act="none", eps_post=1e-6, eps_pre=1e-6, scale=1.0, offset=0.0):
    """((s, bound of s), (x, bound of x) or None).  gate: [T][D], [T][1] or [D]; arrays widened exactly from the bits that the GPU gets."""
    f = lambda a: None if a is None else np.asarray(a, np.float64)  # noqa: E731
    y, gate, r = f(y), f(gate), f(r)
    eps_post, eps_pre, scale, offset = (float(np.float32(a)) for a in (eps_post, eps_pre, scale, offset))
    if y is None:
        s, es = r, np.zeros_like(r)
    else:
        v, ev = normalise(y, np.zeros_like(y), post, f(w_post), f(b_post), offset, eps_post)
        g, rel = np.float64(1.0), 2 * U
        if gate is not None:
            g = gate
            if gate_act == "sigmoid":
                g, rel = 1 / (1 + np.exp(-gate)), (np.abs(gate) + 8) * U
        s = scale * g * v
        es = np.abs(scale * g) * ev + np.abs(s) * (rel + 3 * U)
        if r is not None:
            s = s + r
            es = es + U * np.abs(s)
    if pre == "none":
        return (s, es), None
    return (s, es), normalise(s, es, pre, f(w_pre), f(b_pre), offset, eps_pre)
