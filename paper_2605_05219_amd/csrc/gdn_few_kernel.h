// Products of a few rows with a weight matrix: the part that the projections' and the experts' kernels share.
//
// With at most 64 rows such a product does at most 64 flops for every weight element's 2 bytes: it is bound by how fast the
// weights come from memory, not by the matrix cores.  So nothing is staged: a wave's lanes load weight rows straight into the
// left operand's registers of v_mfma_f32_16x16x32_bf16 (lane: row lane % 16, k 8 (lane / 16) .. + 7: 16 bytes), x rows, which the
// caches hold, into the right one's, and the waves of a workgroup share the k range out step by step, a step of 64 (a whole
// 128-byte line of every row) to a wave, U steps on their way at once.  Their sums meet in LDS, in the order of the waves.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace gdn {
namespace few {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int STEP = 64;                          // k of a step

// acc[i][j] += (weight tile i) x (row tile j) over the wave's share of `steps` k steps.  wp[i], xp[j]: the lane's row of the tile at k = 8 (lane / 16).
// Result: lane lr = lane % 16 holds row lr of tile j, register e output 4 (lane / 16) + e of tile i.
template <int NT, int RT, int WAVES, int U>
__device__ __forceinline__ void accumulate(f32x4 (&acc)[NT][RT], const uint16_t* const (&wp)[NT], const uint16_t* const (&xp)[RT], int steps, int wave) {
    u32x4 w[U][2][NT], x[U][2][RT];
    for (int s0 = wave; s0 < steps; s0 += WAVES * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * WAVES;
            if (s >= steps) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < NT; ++i) w[u][h][i] = *reinterpret_cast<const u32x4*>(wp[i] + s * STEP + 32 * h);
#pragma unroll
                for (int j = 0; j < RT; ++j) x[u][h][j] = *reinterpret_cast<const u32x4*>(xp[j] + s * STEP + 32 * h);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * WAVES >= steps) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < RT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[u][h][i]), __builtin_bit_cast(bf16x8, x[u][h][j]),
                                                                            acc[i][j], 0, 0, 0);
        }
    }
}

// The waves' sums to LDS: [wave][tile i][row of all row tiles][16 outputs], 16-byte pieces.
template <int NT, int RT, int WAVES>
__device__ __forceinline__ void put_sums(f32x4 (&acc)[NT][RT], f32x4* sums, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) sums[((wave * NT + i) * RT * 16 + j * 16 + (lane & 15)) * 4 + (lane >> 4)] = acc[i][j];
}
template <int NT, int RT, int WAVES>
__device__ __forceinline__ f32x4 get_sum(const f32x4* sums, int tile, int row, int piece) {
    f32x4 v = sums[(tile * RT * 16 + row) * 4 + piece];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sums[((w * NT + tile) * RT * 16 + row) * 4 + piece];
    return v;
}

}  // namespace few
}  // namespace gdn
