// Kernels of a mixture of experts (see include/gdn_moe.h): the router's sums, the choice, the experts' two products, the sum of their outputs.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "gdn_act.h"
#include "gdn_few_kernel.h"
#include "gdn_linear_tiles.h"
#include "gdn_moe.h"

namespace gdn {
namespace moe {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int MAX_E = 1024, MAX_K = 16;

struct MoeArgs {
    const uint16_t* x;
    const void* w_router;
    const float* choice_bias;
    const uint16_t *w_gate_up, *w_down, *add;
    uint16_t* y;
    int32_t* out_ids;             // the caller's, or null
    float* out_weights;
    int64_t ldx, ld_add, ldy;
    int32_t T, E, k, D, F;
    int32_t act, score, normalise, router_f32;
    float routed_scale;
    // workspace
    float* logits;                // [T][E]
    int32_t* ids;                 // [T][k]: -1 for a choice that is left out
    float* weights;               // [T][k]
    int32_t* counts;              // [E]: choices of an expert; then the number of experts that have any
    int32_t* active;              // those experts, in no order
    int32_t* list;                // [E][T]: an expert's choices (t k + j), in no order: no result depends on it
    uint16_t* h;                  // [T k][F]
    float* part;                  // [T k][D]: weighted outputs
    linear::ExpertTile* table;    // tiles of tile_rows rows, an expert's one after the other; n_tiles: how many
    int32_t* n_tiles;
    int32_t tile_rows;
};

// ---- the router's sums.  A wave makes TE experts x TT tokens, its lanes along D, 8 elements at a time.  The sums decide a choice, so
// that one in fp32, whose error changes with the order of its terms, would let the choice hang on how the work is split: in fp64 a sum of products of two bf16
// numbers is exact but for terms 2^30 times smaller than the largest, whatever the order, and equal rows of w_router give equal keys.
template <int TT, int TE>
__global__ void __launch_bounds__(256) moe_logits_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (blockIdx.x == 0 && blockIdx.y == 0)                      // the counts of the launch behind this one
        for (int e = threadIdx.x; e <= a.E; e += 256) a.counts[e] = 0;
    const int t0 = blockIdx.y * TT, e0 = (blockIdx.x * 4 + wave) * TE;
    if (e0 >= a.E) return;
    double acc[TE][TT];
#pragma unroll
    for (int i = 0; i < TE; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = 0.0;
    for (int c = 8 * lane; c < a.D; c += 512) {
        float xv[TT][8], wv[TE][8];
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(a.x + (int64_t)min(t0 + j, a.T - 1) * a.ldx + c);
#pragma unroll
            for (int q = 0; q < 4; ++q) { xv[j][2 * q] = __uint_as_float(v[q] << 16); xv[j][2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u); }
        }
#pragma unroll
        for (int i = 0; i < TE; ++i) {
            const int64_t at = (int64_t)min(e0 + i, a.E - 1) * a.D + c;
            if (a.router_f32) {
                const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.w_router) + at);
                const f32x4 lo = p[0], hi = p[1];
#pragma unroll
                for (int q = 0; q < 4; ++q) { wv[i][q] = lo[q]; wv[i][q + 4] = hi[q]; }
            } else {
                const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.w_router) + at);
#pragma unroll
                for (int q = 0; q < 4; ++q) { wv[i][2 * q] = __uint_as_float(v[q] << 16); wv[i][2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u); }
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            double xd[TT], wd[TE];
#pragma unroll
            for (int j = 0; j < TT; ++j) xd[j] = (double)xv[j][q];
#pragma unroll
            for (int i = 0; i < TE; ++i) wd[i] = (double)wv[i][q];
#pragma unroll
            for (int i = 0; i < TE; ++i)
#pragma unroll
                for (int j = 0; j < TT; ++j) acc[i][j] = fma(wd[i], xd[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < TE; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            double v = acc[i][j];
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
            if (lane == 0 && e0 + i < a.E && t0 + j < a.T) a.logits[(int64_t)(t0 + j) * a.E + e0 + i] = (float)v;
        }
}

// ---- the choice, a wave to a token.  Lane l holds the keys of experts P l .. P l + P - 1 as whole numbers of the same order, so that of the lanes with the
// largest key the first has the lowest index.
__device__ __forceinline__ uint32_t key_order(float key) {
    if (key != key) return 1;                                    // a NaN: behind every number that can be chosen
    if (key == -__builtin_inff()) return 0;                      // never chosen
    const uint32_t b = __float_as_uint(key + 0.f);               // (-0 and 0 are equal)
    return (b & 0x80000000u ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ float wave_fmax(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}

// The choices of one token: lane j < k gets the j-th one's expert (-1 where there is none) and weight.
template <int P>
__device__ __forceinline__ void choose(const MoeArgs& a, int t, int lane, int& my_id, float& my_weight) {
    float l[P];
    uint32_t key[P];
    const float* row = a.logits + (int64_t)t * a.E;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int e = lane * P + i;
        l[i] = -__builtin_inff();
        key[i] = 0;
        if (e < a.E) {
            l[i] = row[e];
            float s = l[i];
            if (a.score == GDN_SCORE_SIGMOID || a.choice_bias) {
                double d = a.score == GDN_SCORE_SIGMOID ? 1.0 / (1.0 + exp(-(double)l[i])) : (double)l[i];
                if (a.choice_bias) d += (double)a.choice_bias[e];
                s = (float)d;
            }
            key[i] = key_order(s);
        }
    }
    float top = 0.f, total = 1.f;
    if (a.score == GDN_SCORE_SOFTMAX && !a.normalise) {          // over all experts
        float m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < P; ++i) m = fmaxf(m, l[i]);
        top = wave_fmax(m);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (lane * P + i < a.E) s += expf(l[i] - top);
        total = wave_sum(s);
    }
    my_id = -1;
    float my_l = 0.f;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) best = max(best, key[i]);
        const uint32_t most = wave_max(best);
        if (most == 0) break;
        const int first = __ffsll((unsigned long long)__ballot(best == most)) - 1;
        int at = 0;
        float at_l = 0.f;
        bool found = false;
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (!found && key[i] == most) {
                found = true;
                at = lane * P + i;
                at_l = l[i];
                if (lane == first) key[i] = 0;
            }
        at = __shfl(at, first);
        at_l = __shfl(at_l, first);
        if (lane == j) { my_id = at; my_l = at_l; }
    }
    float p = 0.f;
    const bool have = lane < a.k && my_id >= 0;
    if (a.score == GDN_SCORE_SOFTMAX) {
        if (a.normalise) top = wave_fmax(have ? my_l : -__builtin_inff());
        if (have) p = expf(my_l - top);
        if (!a.normalise) p = p / total;
    } else if (have) {
        p = 1.f / (1.f + expf(-my_l));
    }
    if (a.normalise) {
        const float sum = wave_sum(p);
        p = sum == 0.f ? 0.f : p / sum;
    }
    my_weight = have ? p * a.routed_scale : 0.f;
}

template <int P>
__global__ void __launch_bounds__(256) moe_route_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63;
    const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    int id;
    float p;
    choose<P>(a, t, lane, id, p);
    if (lane >= a.k) return;
    const int pair = t * a.k + lane;
    if (a.out_ids) a.out_ids[pair] = id;
    if (a.out_weights) a.out_weights[pair] = p;
    const bool in = id >= 0 && p != 0.f;                         // (a NaN weight is in)
    a.ids[pair] = in ? id : -1;
    a.weights[pair] = p;
    if (in) {
        const int at = atomicAdd(a.counts + id, 1);
        a.list[(int64_t)id * a.T + at] = pair;
        if (at == 0) a.active[atomicAdd(a.counts + a.E, 1)] = id;
    }
}

// ---- the tile table, one workgroup: thread e has expert e's tiles, and those of the experts before it by a sum over the threads
__global__ void __launch_bounds__(MAX_E) moe_tiles_kernel(MoeArgs a) {
    __shared__ int32_t before[MAX_E / 64];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const int n = e < a.E ? a.counts[e] : 0, tiles = (n + a.tile_rows - 1) / a.tile_rows;
    int sum = tiles;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(sum, m);
        if (lane >= m) sum += other;
    }
    if (lane == 63) before[wave] = sum;
    __syncthreads();
    int first = sum - tiles;
    for (int w = 0; w < wave; ++w) first += before[w];
    for (int i = 0; i < tiles; ++i) a.table[first + i] = linear::ExpertTile{e, first, tiles, n};
    if (e == MAX_E - 1) *a.n_tiles = first + tiles;
}

// ---- h = act(gate x) * (up x): a workgroup makes 16 of an expert's F for all of its rows, 16 RT at a time
constexpr int UP_WAVES = 8;
template <int RT>
__global__ void __launch_bounds__(64 * UP_WAVES) moe_up_kernel(MoeArgs a) {
    constexpr int U = RT == 4 ? 2 : 4;
    __shared__ f32x4 sums[UP_WAVES * 2 * RT * 16 * 4];
    __shared__ int32_t rows[RT * 16];
    if ((int)blockIdx.y >= a.counts[a.E]) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, g = lane >> 4;
    const int e = a.active[blockIdx.y], n = a.counts[e], f0 = blockIdx.x * 16;
    const int32_t* list = a.list + (int64_t)e * a.T;
    const uint16_t* wp[2];
    wp[0] = a.w_gate_up + ((int64_t)e * 2 * a.F + f0 + lr) * a.D + 8 * g;
    wp[1] = wp[0] + (int64_t)a.F * a.D;
    for (int r0 = 0; r0 < n; r0 += 16 * RT) {
        if (threadIdx.x < RT * 16) rows[threadIdx.x] = list[min(r0 + (int)threadIdx.x, n - 1)];
        __syncthreads();
        const uint16_t* xp[RT];
        f32x4 acc[2][RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            xp[j] = a.x + (int64_t)(rows[16 * j + lr] / a.k) * a.ldx + 8 * g;
            acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        few::accumulate<2, RT, UP_WAVES, U>(acc, wp, xp, a.D / few::STEP, wave);
        few::put_sums<2, RT, UP_WAVES>(acc, sums, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < RT * 16 * 4; i += 64 * UP_WAVES) {
            const int row = i >> 2, piece = i & 3;
            if (r0 + row >= n) continue;
            f32x4 v = activate(a.act, few::get_sum<2, RT, UP_WAVES>(sums, 0, row, piece));
            v *= few::get_sum<2, RT, UP_WAVES>(sums, 1, row, piece);
            *reinterpret_cast<bf16x4*>(a.h + (int64_t)rows[row] * a.F + f0 + 4 * piece) = __builtin_convertvector(v, bf16x4);
        }
        __syncthreads();
    }
}

// ---- part = weight * (w_down h): a workgroup makes 16 of D for all of an expert's rows
constexpr int DOWN_WAVES = 4;
template <int RT>
__global__ void __launch_bounds__(64 * DOWN_WAVES) moe_down_kernel(MoeArgs a) {
    constexpr int U = RT == 4 ? 2 : 4;
    __shared__ f32x4 sums[DOWN_WAVES * RT * 16 * 4];
    __shared__ int32_t rows[RT * 16];
    if ((int)blockIdx.y >= a.counts[a.E]) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, g = lane >> 4;
    const int e = a.active[blockIdx.y], n = a.counts[e], d0 = blockIdx.x * 16;
    const int32_t* list = a.list + (int64_t)e * a.T;
    const uint16_t* wp[1] = {a.w_down + ((int64_t)e * a.D + d0 + lr) * a.F + 8 * g};
    for (int r0 = 0; r0 < n; r0 += 16 * RT) {
        if (threadIdx.x < RT * 16) rows[threadIdx.x] = list[min(r0 + (int)threadIdx.x, n - 1)];
        __syncthreads();
        const uint16_t* xp[RT];
        f32x4 acc[1][RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            xp[j] = a.h + (int64_t)rows[16 * j + lr] * a.F + 8 * g;
            acc[0][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        few::accumulate<1, RT, DOWN_WAVES, U>(acc, wp, xp, a.F / few::STEP, wave);
        few::put_sums<1, RT, DOWN_WAVES>(acc, sums, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < RT * 16 * 4; i += 64 * DOWN_WAVES) {
            const int row = i >> 2, piece = i & 3;
            if (r0 + row >= n) continue;
            *reinterpret_cast<f32x4*>(a.part + (int64_t)rows[row] * a.D + d0 + 4 * piece) =
                a.weights[rows[row]] * few::get_sum<1, RT, DOWN_WAVES>(sums, 0, row, piece);
        }
        __syncthreads();
    }
}

// ---- y = add + the choices' parts, in the order of their keys; a thread owns 8 adjacent channels
__global__ void __launch_bounds__(256) moe_sum_kernel(MoeArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int groups = a.D / 8;
    if (i >= (int64_t)a.T * groups) return;
    const int t = (int)(i / groups), c = (int)(i % groups) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.add) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(a.add + (int64_t)t * a.ld_add + c);
#pragma unroll
        for (int q = 0; q < 4; ++q) { v[2 * q] = __uint_as_float(r[q] << 16); v[2 * q + 1] = __uint_as_float(r[q] & 0xffff0000u); }
    }
    for (int j = 0; j < a.k; ++j) {
        const int64_t pair = (int64_t)t * a.k + j;
        if (a.ids[pair] < 0) continue;
        const f32x4* p = reinterpret_cast<const f32x4*>(a.part + pair * a.D + c);
        const f32x4 lo = p[0], hi = p[1];
#pragma unroll
        for (int q = 0; q < 4; ++q) { v[q] += lo[q]; v[q + 4] += hi[q]; }
    }
    bf16x8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (__bf16)v[q];
    *reinterpret_cast<bf16x8*>(a.y + (int64_t)t * a.ldy + c) = o;
}

}  // namespace moe
}  // namespace gdn
