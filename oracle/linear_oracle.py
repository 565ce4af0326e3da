"""Oracle of the layer's projections.  TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product path,
and it shares no code with the HIP library.

The paper times a layer group of GatedDeltaNet and attention layers (Sec. 6, prototype wall-clock time) and does not
restate the layers; their projections are the plain affine maps of any such layer,
    y[t][n] = bias[n] + sum_k x[t][k] w[n][k]          (weights stored [out][in]),
written out here as the definition: an explicit triple loop in fp64 for small cases, and the same sum through
numpy's fp64 matrix product for the sizes the parity tests use.  Inputs are the bits the GPU gets (bf16 carried as
uint16, or fp32), widened exactly to fp64.

Pins (tests/test_linear_oracle_pins.py): the two forms against each other, a hand-worked case, the identity and a
permutation matrix, linearity, the bias alone, and the [out][in] storage convention.
"""
from __future__ import annotations

import numpy as np


def _f64(a) -> np.ndarray:
    a = np.asarray(a)
    if a.dtype == np.uint16:                       # bf16 bit patterns
        return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def linear_loops(x, w, bias=None) -> np.ndarray:
    """The definition, term by term (small inputs only)."""
    x, w = _f64(x), _f64(w)
    T, K = x.shape
    N, K2 = w.shape
    assert K == K2
    b = np.zeros(N) if bias is None else _f64(bias)
    y = np.zeros((T, N), dtype=np.float64)
    for t in range(T):
        for n in range(N):
            acc = b[n]
            for k in range(K):
                acc += x[t, k] * w[n, k]
            y[t, n] = acc
    return y


def linear(x, w, bias=None) -> np.ndarray:
    """The same sum through the fp64 matrix product (rounding order aside)."""
    x, w = _f64(x), _f64(w)
    y = x @ w.T
    if bias is not None:
        y = y + _f64(bias)[None, :]
    return y


def _erf(z):
    from scipy.special import erf
    return erf(z)


ACTS = {
    "none": lambda z: z,
    "silu": lambda z: z / (1 + np.exp(-z)),
    "gelu": lambda z: 0.5 * z * (1 + _erf(z / np.sqrt(2))),
    "gelu_tanh": lambda z: 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))),
    "relu": lambda z: np.maximum(z, 0),
    "relu2": lambda z: np.maximum(z, 0) ** 2,
    "sigmoid": lambda z: 1 / (1 + np.exp(-z)),
}
EPS23 = 2.0 ** -23


def act_with_bound(act, z, ez):
    """(act(z), bound of the error of an fp32 evaluation at a z that is off by at most ez).  The slopes of the smooth activations are at most 1.13; an
    exponential in fp32 is off by a relative (its argument + 4) 2^-23, sums, reciprocals and products by 2^-23 each; erf by 2^-22."""
    a = ACTS[act](z)
    if act in ("none", "relu"):
        return a, ez
    if act == "relu2":
        return a, 2 * np.abs(z) * ez + ez * ez + EPS23 * np.abs(a)
    if act == "sigmoid":
        return a, 0.25 * ez + (np.abs(z) + 12) * EPS23 * a
    if act == "gelu":
        return a, 1.13 * ez + 4 * EPS23 * np.abs(z)
    arg = np.abs(z) if act == "silu" else 1.6 * (np.abs(z) + 0.045 * np.abs(z) ** 3)
    # (where the exponential overflows the value is the product with zero; the bound's floor is the least normal number)
    return a, 1.13 * ez + (4 * arg + 16) * EPS23 * np.abs(a) + 2.0 ** -126


def linear_act(x, w, bias, act="none", w_up=None, bias_up=None, residual=None, scale=1.0):
    """(y, bound of fp32's error) of y = scale * act(x w^T + bias) [* (x w_up^T + bias_up)] + residual.  A product of two bf16 numbers is exact in fp32; a sum
    of K of them is off by at most K 2^-23 sum |x w| (one unit for an addition covers a matrix core that truncates)."""
    def product(w, b):
        z = linear(x, w, b)
        e = (_f64(x).shape[1] + 8) * EPS23 * linear(np.abs(_f64(x)), np.abs(_f64(w)))
        return z, e + EPS23 * np.abs(z)
    a, ea = act_with_bound(act, *product(w, bias))
    if w_up is not None:
        up, eu = product(w_up, bias_up)
        a, ea = a * up, ea * np.abs(up) + np.abs(a) * eu + ea * eu + EPS23 * np.abs(a * up)
    scale = float(np.float32(scale))
    y, ey = scale * a, abs(scale) * ea + EPS23 * np.abs(scale * a)
    if residual is not None:
        y = y + _f64(residual)
        ey = ey + EPS23 * np.abs(y)
    return y, ey
