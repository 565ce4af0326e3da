// The activations of the products' epilogues.
#pragma once
#include <hip/hip_runtime.h>

#include "gdn_linear.h"

namespace gdn {

typedef float act_f32x4 __attribute__((ext_vector_type(4)));

// z Phi(z), Phi(-|z|) = P(t) t exp(-z^2 / 2) and Phi(|z|) = 1 - Phi(-|z|), with t = 1 / (1 + 0.33 |z| / sqrt 2).  P is the polynomial of degree 7 that is off by the least relative error from
// exp(x^2) erfc(x) / (2 t), x = |z| / sqrt 2 from 0 to 9.8 (exchange of its extremes, in 64 bits: 8.6e-8; 4 units of 2^-23 with the roundings of its terms in fp32), which goes to
// 0.33 / (2 sqrt pi) as t goes to 0, so that the far negative side keeps its digits: (0.6 z^2 + 8) 2^-23 of the value, the first part from rounding the exponential's argument; a
// polynomial for an absolute error of erfc loses them (1.5e-7 absolute: 5e-4 of the value at -4, 1e-2 at -8).  Values below 2^-126 may be zero.  No branch, and no more time than
// that one (1401 x 1733 x 1600 onto an fp32 residual 20.6 us with either).
__device__ __forceinline__ float gelu(float z) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.33f * 0.70710678118654752f, fabsf(z), 1.f));
    float q = fmaf(t, -0.0678544938f, 0.230882104f);
    q = fmaf(t, q, -0.176910717f);
    q = fmaf(t, q, 0.205508224f);
    q = fmaf(t, q, 0.0229227514f);
    q = fmaf(t, q, 0.10082951f);
    q = fmaf(t, q, 0.0914411187f);
    q = fmaf(t, q, 0.0931814766f);
    q *= t * __builtin_amdgcn_exp2f(-0.72134752044448170f * (z * z));      // 1 / (2 ln 2)
    return z < 0.f ? z * q : z < 1e30f ? z - z * q : z;          // (q is zero from 14 on, and an infinity times zero no number)
}

// f(z) of four values in fp32.  The reciprocal is the hardware's, off by 2^-23; so is the exponential, whose argument is rounded when it is multiplied by log2 e: off by a
// relative (|argument| + 2) 2^-23, some 2^-17 at 80, and so are the values that are an exponential far out (SiLU and sigmoid of a z far below zero; GELU by tanh with u for the argument, which
// has three roundings more).  Values below 2^-126 may be zero.  A NaN stays a NaN.  `act` is the same on every lane, so the choice is a scalar branch.
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
