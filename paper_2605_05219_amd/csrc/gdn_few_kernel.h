// A product of a few rows with a weight matrix, for the projections' epilogues.
//
// With a few rows such a product does few flops for every weight element's 2 bytes: it is bound by how fast the weights come from
// memory, and with the few workgroups that a narrow output gives, by how much of them each has on its way.  The tiles of gdn_linear.hip
// walk k one step after the other, with a barrier each (0.13 to 0.2 us a step: 96 steps of a 2048 x 6144 weight take 17 us at best); here the waves of a
// workgroup share the steps out instead.  A wave has a ring of its own in LDS, which 16-byte loads to LDS fill S steps of 64 ahead, and no other wave
// reads it: there is no barrier until the waves' sums meet, in LDS, in the order of the waves.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gdn_few_parts.h"

namespace gdn {
namespace few {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// RT: tiles of 16 rows of x; WR: weight rows of a workgroup (8, 16 or 32); WAVES waves; S steps of a wave on their way
template <int RT_, int WR_, int WAVES_, int S_>
struct Few {
    static constexpr int RT = RT_, WR = WR_, WAVES = WAVES_, S = S_, ROWS = 16 * RT;
    static constexpr int CT = (WR + 15) / 16;     // tiles of 16 weight rows (of 8 rows the tile's other half is what lies behind them in LDS, for sums that go nowhere)
    static constexpr int X_LOADS = ROWS / 8, W_LOADS = WR / 8, LOADS = X_LOADS + W_LOADS;        // of 1 KiB, 8 rows each, per step
    static constexpr int HALF = (W_LOADS + 1) / 2;                                               // the first part's loads of the weights
    static constexpr int STAGE = LOADS * 1024, RING = S * STAGE;
    static constexpr int SUMS = CT * ROWS * 64;   // bytes of a wave's sums: [tile][row][16 outputs]
    static constexpr int SMEM = WAVES * (RING > SUMS ? RING : SUMS) + (WR == 8 ? 1024 : 0);
    static constexpr int AHEAD = (S - 1) * LOADS; // loads that may be on their way when a step's have landed
    static_assert(SMEM <= 160 * 1024 && AHEAD < 64, "ring");

    // One step's loads, k bytes on in the rows.  They go out for every step slot, also behind the last one (not live, an empty descriptor: nothing is fetched), so
    // that the number on their way, and with it the wait, is always the same.
    static __device__ __forceinline__ void fetch(char* to, int k, const Part& w0, const Part& w1, const Part& x, bool live, const int* xoff, const int* woff) {
#pragma unroll
        for (int j = 0; j < W_LOADS; ++j) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(j >= HALF ? w1.at : w0.at), 0, live ? (j >= HALF ? w1.bytes : w0.bytes) : 0, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + (X_LOADS + j) * 1024), 16, woff[j], k, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(x.at), 0, live ? x.bytes : 0, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + j * 1024), 16, xoff[j], k, 0, 0);
        }
    }

    // The sums of a wave's steps over the weight rows, w0's (8 HALF) and then w1's, and rows x.  acc[i RT + j]: lane lr = lane % 16 holds row lr of row tile j,
    // register e weight row 16 i + 4 (lane / 16) + e.  place(step, w0, w1, x) moves the parts to a step's rows (those of another matrix of the same pitch, for
    // one) and returns its bytes along k.
    template <typename PLACE>
    static __device__ __forceinline__ void sums_of(f32x4* acc, const Part& w0, const Part& w1, const Part& x, int steps, PLACE place, char* ring, int wave, int lane) {
        const int row = lane >> 3, pos = lane & 7;    // of a load: lane i lands at row i / 8, piece i % 8
        int xoff[X_LOADS], woff[W_LOADS];
#pragma unroll
        for (int j = 0; j < X_LOADS; ++j) xoff[j] = load_offset(8 * j + row, 8 * j + row, pos, x.pitch);
#pragma unroll
        for (int j = 0; j < W_LOADS; ++j) woff[j] = load_offset(8 * j + row, 8 * (j >= HALF ? j - HALF : j) + row, pos, j >= HALF ? w1.pitch : w0.pitch);
        auto load = [&](int slot, int step) {
            Part v0 = w0, v1 = w1, vx = x;
            const bool live = step < steps;
            const int k = live ? place(step, v0, v1, vx) : 0;
            fetch(ring + slot * STAGE, k, v0, v1, vx, live, xoff, woff);
        };
#pragma unroll
        for (int s = 0; s < S; ++s) load(s, wave + s * WAVES);
        const int lr = lane & 15, g = lane >> 4, sw = lr >> 1;
        int slot = 0;
        for (int step = wave; step < steps; step += WAVES) {
            __builtin_amdgcn_s_waitcnt(((AHEAD & 0x30) << 10) | (AHEAD & 0xF) | 0x0F70);      // this step's loads have landed (vmcnt)
            asm volatile("" ::: "memory");
            const char* at = ring + slot * STAGE + lr * 128;
            u32x4 wf[2][CT], xf[2][RT];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int piece = ((4 * h + g) ^ sw) << 4;
#pragma unroll
                for (int i = 0; i < CT; ++i) wf[h][i] = *reinterpret_cast<const u32x4*>(at + X_LOADS * 1024 + i * 2048 + piece);
#pragma unroll
                for (int j = 0; j < RT; ++j) xf[h][j] = *reinterpret_cast<const u32x4*>(at + j * 2048 + piece);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);       // read (lgkmcnt(0)): the slot is free
            asm volatile("" ::: "memory");
            load(slot, step + S * WAVES);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < CT; ++i)
#pragma unroll
                    for (int j = 0; j < RT; ++j)
                        acc[i * RT + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wf[h][i]), __builtin_bit_cast(bf16x8, xf[h][j]),
                                                                                  acc[i * RT + j], 0, 0, 0);
            slot = slot + 1 == S ? 0 : slot + 1;
        }
    }

    // The waves' sums to LDS (behind a barrier of the caller's: the rings have been read), and one of them.
    static __device__ __forceinline__ void put_sums(const f32x4* acc, f32x4* sums, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int j = 0; j < RT; ++j) sums[((wave * CT + i) * ROWS + j * 16 + (lane & 15)) * 4 + (lane >> 4)] = acc[i * RT + j];
    }
    static __device__ __forceinline__ f32x4 get_sum(const f32x4* sums, int row, int quad) {      // weight rows 4 quad .. + 3
        const int at = ((quad >> 2) * ROWS + row) * 4 + (quad & 3);
        f32x4 v = sums[at];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w * CT * ROWS * 4 + at];
        return v;
    }
};

}  // namespace few
}  // namespace gdn
