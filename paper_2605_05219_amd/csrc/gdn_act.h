// The activations of the products' epilogues.
#pragma once
#include <hip/hip_runtime.h>

#include "gdn_linear.h"

namespace gdn {

typedef float act_f32x4 __attribute__((ext_vector_type(4)));

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
            for (int e = 0; e < 4; ++e) z[e] = 0.5f * z[e] * (1.f + erff(z[e] * 0.70710678118654752f));
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
