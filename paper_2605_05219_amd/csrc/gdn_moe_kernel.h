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
    int32_t* counts;              // [E]: choices of an expert
    int32_t* list;                // [E][T]: an expert's choices (t k + j)
    uint16_t* h;                  // [T k][F]: weighted
    float* part;                  // [T k][D]: the choices' outputs
    linear::ExpertTile* table;    // tiles of tile_rows rows, an expert's one after the other; n_tiles: how many
    int32_t* n_tiles;
    int32_t tile_rows;
};

// Sums and largest values over a wave, by moves within the vector unit (a shuffle goes through LDS: 64 of them are what a choice would wait for).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t none) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}
// Lane 63 gets op over all lanes: 1, 2, 4, 8 lanes up within a row of 16, then the last lane of a row to the next row, and of the first half to the second.
template <typename T, typename OP>
__device__ __forceinline__ T wave_up(T v, uint32_t none, OP op) {
    v = op(v, __builtin_bit_cast(T, moved<0x111, 0xf>(__builtin_bit_cast(uint32_t, v), none)));
    v = op(v, __builtin_bit_cast(T, moved<0x112, 0xf>(__builtin_bit_cast(uint32_t, v), none)));
    v = op(v, __builtin_bit_cast(T, moved<0x114, 0xf>(__builtin_bit_cast(uint32_t, v), none)));
    v = op(v, __builtin_bit_cast(T, moved<0x118, 0xf>(__builtin_bit_cast(uint32_t, v), none)));
    v = op(v, __builtin_bit_cast(T, moved<0x142, 0xa>(__builtin_bit_cast(uint32_t, v), none)));
    v = op(v, __builtin_bit_cast(T, moved<0x143, 0xc>(__builtin_bit_cast(uint32_t, v), none)));
    return v;
}
template <typename T>
__device__ __forceinline__ T from_lane(T v, int lane) { return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { return from_lane(wave_up(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }), 63); }
__device__ __forceinline__ float wave_sum(float v) { return from_lane(wave_up(v, 0u, [](float a, float b) { return a + b; }), 63); }
__device__ __forceinline__ float wave_fmax(float v) { return from_lane(wave_up(v, 0xff800000u, [](float a, float b) { return fmaxf(a, b); }), 63); }
// The sum of fp64 values, on lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_add(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t m = (uint64_t)moved<CTRL, ROWS>((uint32_t)(b >> 32), 0) << 32 | moved<CTRL, ROWS>((uint32_t)b, 0);
    return v + __builtin_bit_cast(double, m);
}
__device__ __forceinline__ double wave_total(double v) {
    v = moved_add<0x111, 0xf>(v);
    v = moved_add<0x112, 0xf>(v);
    v = moved_add<0x114, 0xf>(v);
    v = moved_add<0x118, 0xf>(v);
    v = moved_add<0x142, 0xa>(v);
    return moved_add<0x143, 0xc>(v);
}

// ---- the router's sums.  The sums decide a choice, so that one in fp32, whose error changes with the order of its terms, would let the choice hang on how the
// work is split: in fp64 a sum of products of two bf16 numbers is exact but for terms 2^30 times smaller than the largest, whatever the order, and equal rows of
// w_router give equal keys.
//
// Few tokens: a wave makes TE experts x TT tokens, its lanes along D, 8 elements at a time, U such pieces of a row on their way at once: the time is the latency of
// its loads and of the conversions behind them, so that few sums are given a wave each (1 token x 128 experts, D 2048: 3.7 us, 5.0 with two experts to a wave;
// 64 x 128 7.1 with two tokens to a wave, 7.5 with two of each).
template <int TT, int TE, int U>
__global__ void __launch_bounds__(256) moe_logits_few_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = blockIdx.y * TT, e0 = (blockIdx.x * 4 + wave) * TE;
    if (e0 >= a.E) return;
    double acc[TE][TT];
#pragma unroll
    for (int i = 0; i < TE; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = 0.0;
    const uint16_t* xp[TT];
    int64_t wp[TE];                                              // (rows past the end are the last one's: their sums go nowhere)
#pragma unroll
    for (int j = 0; j < TT; ++j) xp[j] = a.x + (int64_t)min(t0 + j, a.T - 1) * a.ldx;
#pragma unroll
    for (int i = 0; i < TE; ++i) wp[i] = (int64_t)min(e0 + i, a.E - 1) * a.D;
    for (int c0 = 8 * lane; c0 < a.D; c0 += 512 * U) {
        u32x4 xr[U][TT], wr[U][TE][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + 512 * u;
            const bool in = c < a.D;
#pragma unroll
            for (int j = 0; j < TT; ++j) xr[u][j] = in ? *reinterpret_cast<const u32x4*>(xp[j] + c) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < TE; ++i) {
                wr[u][i][0] = wr[u][i][1] = u32x4{0, 0, 0, 0};
                if (!in) continue;
                if (a.router_f32) {
                    const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(a.w_router) + wp[i] + c);
                    wr[u][i][0] = p[0];
                    wr[u][i][1] = p[1];
                } else {
                    wr[u][i][0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.w_router) + wp[i] + c);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                double xd[TT], wd[TE];
#pragma unroll
                for (int j = 0; j < TT; ++j) xd[j] = (double)__uint_as_float(q & 1 ? xr[u][j][q / 2] & 0xffff0000u : xr[u][j][q / 2] << 16);
#pragma unroll
                for (int i = 0; i < TE; ++i)
                    wd[i] = (double)__uint_as_float(a.router_f32 ? wr[u][i][q / 4][q % 4] : q & 1 ? wr[u][i][0][q / 2] & 0xffff0000u : wr[u][i][0][q / 2] << 16);
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
            const double v = wave_total(acc[i][j]);
            if (lane == 63 && e0 + i < a.E && t0 + j < a.T) a.logits[(int64_t)(t0 + j) * a.E + e0 + i] = (float)v;
        }
}

// More: a workgroup makes 16 experts x 16 tokens on v_mfma_f64_16x16x4_f64 (lane: row lane % 16 of either operand and one k of its group of 16 lanes; of the result
// token lane % 16, register r expert lane / 16 + 4 r), its waves the blocks of 32 k in turn: a lane loads 8 adjacent elements of each row, and which k a product
// pairs is the same for both.  Making fp64 of the elements is what the vector units spend most on, and a matrix product takes sixteen uses of each: 200 tokens x 512
// experts, D 2048, 17 us, 2048 x 64 17.5 (by 4 x 4 on the vector units 27 and 35; 1 x 128 8.5, 64 x 128 9.6 against 3.7 and 7.1 of the kernel above).
template <int WAVES>
__global__ void __launch_bounds__(64 * WAVES) moe_logits_kernel(MoeArgs a) {
    typedef double f64x4 __attribute__((ext_vector_type(4)));
    __shared__ f64x4 sums[WAVES][64];
    constexpr int U = 4;                                          // blocks on their way
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, g = lane >> 4;
    const int t0 = blockIdx.x * 16, e0 = blockIdx.y * 16;      // (the tokens may be more than a grid's y holds)
    // (rows past the end are the last one's: their sums go nowhere)
    const uint16_t* const x = a.x + (int64_t)min(t0 + lr, a.T - 1) * a.ldx + 8 * g;
    const int64_t w = (int64_t)min(e0 + lr, a.E - 1) * a.D + 8 * g;
    f64x4 acc = {0.0, 0.0, 0.0, 0.0};
    const int blocks = a.D / 32;
    for (int b0 = wave; b0 < blocks; b0 += WAVES * U) {
        u32x4 xr[U], wr[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = b0 + u * WAVES;
            xr[u] = wr[u][0] = wr[u][1] = u32x4{0, 0, 0, 0};
            if (b >= blocks) continue;
            xr[u] = *reinterpret_cast<const u32x4*>(x + 32 * b);
            if (a.router_f32) {
                const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(a.w_router) + w + 32 * b);
                wr[u][0] = p[0];
                wr[u][1] = p[1];
            } else {
                wr[u][0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.w_router) + w + 32 * b);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b0 + u * WAVES >= blocks) break;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const uint32_t half = q & 1 ? wr[u][0][q / 2] & 0xffff0000u : wr[u][0][q / 2] << 16;
                const float wv = __uint_as_float(a.router_f32 ? wr[u][q / 4][q % 4] : half);
                const float xv = __uint_as_float(q & 1 ? xr[u][q / 2] & 0xffff0000u : xr[u][q / 2] << 16);
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)wv, (double)xv, acc, 0, 0, 0);
            }
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (threadIdx.x >= 256) return;
    const int from = threadIdx.x >> 2, r = threadIdx.x & 3;
    double v = sums[0][from][r];
    for (int i = 1; i < WAVES; ++i) v += sums[i][from][r];
    const int t = t0 + (from & 15), e = e0 + (from >> 4) + 4 * r;
    if (t < a.T && e < a.E) a.logits[(int64_t)t * a.E + e] = (float)v;
}

// ---- the choice, a wave to a token.  Lane l holds the keys of experts P l .. P l + P - 1 as whole numbers of the same order, so that of the lanes with the
// largest key the first has the lowest index.
__device__ __forceinline__ uint32_t key_order(float key) {
    if (key != key) return 1;                                    // a NaN: behind every number that can be chosen
    if (key == -__builtin_inff()) return 0;                      // never chosen
    const uint32_t b = __float_as_uint(key + 0.f);               // (-0 and 0 are equal)
    return (b & 0x80000000u ? ~b : b | 0x80000000u);
}
// The choices of one token: lane j < k gets the j-th one's expert (-1 where there is none) and weight.
template <int P>
__device__ __forceinline__ void choose(const MoeArgs& a, int t, int lane, int& my_id, float& my_weight) {
    float l[P];
    uint32_t key[P];
    const float* row = a.logits + (int64_t)t * a.E;
    float bias[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {                                // (all asked for before the first is used)
        const int e = min(lane * P + i, a.E - 1);
        l[i] = row[e];
        bias[i] = a.choice_bias ? a.choice_bias[e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float s = l[i];
        if (a.score == GDN_SCORE_SIGMOID || a.choice_bias) {
            double d = a.score == GDN_SCORE_SIGMOID ? 1.0 / (1.0 + exp(-(double)l[i])) : (double)l[i];
            if (a.choice_bias) d += (double)bias[i];
            s = (float)d;
        }
        key[i] = key_order(s);
        if (lane * P + i >= a.E) {
            l[i] = -__builtin_inff();
            key[i] = 0;
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
        at = from_lane(at, first);
        at_l = from_lane(at_l, first);
        if (lane == j) { my_id = at; my_l = at_l; }
    }
    float p = 0.f;
    const bool have = lane < a.k && my_id >= 0;
    if (a.score == GDN_SCORE_SOFTMAX) {
        if (a.normalise) top = wave_fmax(have ? my_l : -__builtin_inff());
        if (have) p = expf(my_l - top);
        if (!a.normalise) p = p / total;
    } else {
        // below -64 a sigmoid is e^l to 2^-92: where the largest of the chosen is there and they are divided by their sum, all of them times e^-largest, so that none that
        // counts is lost to fp32's range (from -88 on 1 / (1 + e^-l) is zero)
        float from = a.normalise ? wave_fmax(have ? my_l : -__builtin_inff()) : 0.f;
        if (!(from < -64.f) || from == -__builtin_inff()) from = 0.f;
        if (have) p = my_l < -64.f ? expf(my_l - from) : 1.f / (1.f + expf(-my_l));
    }
    if (a.normalise) {
        const float sum = wave_sum(p);
        p = sum == 0.f ? 0.f : p / sum;
    }
    my_weight = have ? p * a.routed_scale : 0.f;
}

// The choices of a token to memory; the id that is kept is -1 for a choice of weight zero (a NaN weight is in).
template <int P>
__device__ __forceinline__ void choose_and_keep(const MoeArgs& a, int t, int lane, int32_t* kept) {
    int id;
    float p;
    choose<P>(a, t, lane, id, p);
    if (lane >= a.k) return;
    const int pair = t * a.k + lane;
    if (a.out_ids) a.out_ids[pair] = id;
    if (a.out_weights) a.out_weights[pair] = p;
    const int in = p != 0.f ? id : -1;
    a.ids[pair] = in;
    a.weights[pair] = p;
    if (kept) kept[pair] = in;
}

// The tile table, by a workgroup of MAX_E threads: thread e has expert e's tiles, and those of the experts before it by a sum over the threads.
__device__ __forceinline__ void make_table(const MoeArgs& a, int n, int32_t* before) {
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const int tiles = (n + a.tile_rows - 1) / a.tile_rows;
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

// Few tokens: choices, lists and tile table in one workgroup, a wave to a token.  An expert's list is in no order there: a row of a product
// is the same whatever rows stand beside it.
constexpr int FEW_TOKENS = 16;
template <int P>
__global__ void __launch_bounds__(MAX_E) moe_route_few_kernel(MoeArgs a) {
    __shared__ int32_t kept[FEW_TOKENS * MAX_K], counts[MAX_E], before[MAX_E / 64];
    const int tid = threadIdx.x;
    counts[tid] = 0;
    for (int t = tid >> 6; t < a.T; t += MAX_E / 64) choose_and_keep<P>(a, t, tid & 63, kept);
    __syncthreads();
    if (tid < a.T * a.k) {
        const int e = kept[tid];
        if (e >= 0) a.list[(int64_t)e * a.T + atomicAdd(counts + e, 1)] = tid;
    }
    __syncthreads();
    make_table(a, counts[tid], before);
}

// More: the choices, a wave to a token ...
template <int P>
__global__ void __launch_bounds__(256) moe_route_kernel(MoeArgs a) {
    const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t < a.T) choose_and_keep<P>(a, t, threadIdx.x & 63, nullptr);
}
// ... the lists and the table of a moderate number of choices, in one workgroup ...
constexpr int FEW_PAIRS = 4096;
__global__ void __launch_bounds__(MAX_E) moe_lists_few_kernel(MoeArgs a) {
    __shared__ int32_t counts[MAX_E], before[MAX_E / 64];
    const int tid = threadIdx.x, pairs = a.T * a.k;
    int id[FEW_PAIRS / MAX_E];
#pragma unroll
    for (int i = 0; i < FEW_PAIRS / MAX_E; ++i) id[i] = tid + i * MAX_E < pairs ? a.ids[tid + i * MAX_E] : -1;
    counts[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FEW_PAIRS / MAX_E; ++i)
        if (id[i] >= 0) a.list[(int64_t)id[i] * a.T + atomicAdd(counts + id[i], 1)] = tid + i * MAX_E;
    __syncthreads();
    make_table(a, counts[tid], before);
}
// ... of more the lists, a workgroup to an expert, which looks through all choices (a counter that the tokens of all workgroups add to is
// slower: 12288 choices of 64 experts 37 us, 7 so) ...
constexpr int LIST_WAVES = 16;
__global__ void __launch_bounds__(64 * LIST_WAVES) moe_lists_kernel(MoeArgs a) {
    __shared__ int32_t found[LIST_WAVES];
    const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.T * a.k;
    int32_t* list = a.list + (int64_t)e * a.T;
    int n = 0;
    for (int p0 = 0; p0 < pairs; p0 += 256 * LIST_WAVES) {       // four to a thread
        const int p = p0 + 4 * threadIdx.x;
        int id[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            id[i] = p + i < pairs ? a.ids[p + i] : -1;
            mine += id[i] == e;
        }
        int sum = mine;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        __syncthreads();
        if (lane == 63) found[wave] = sum;
        __syncthreads();
        int at = n + sum - mine;
        for (int w = 0; w < wave; ++w) at += found[w];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (id[i] == e) list[at++] = p + i;
#pragma unroll
        for (int w = 0; w < LIST_WAVES; ++w) n += found[w];
    }
    if (threadIdx.x == 0) a.counts[e] = n;
}
// ... and the tile table.
__global__ void __launch_bounds__(MAX_E) moe_table_kernel(MoeArgs a) {
    __shared__ int32_t before[MAX_E / 64];
    const int e = threadIdx.x;
    make_table(a, e < a.E ? a.counts[e] : 0, before);
}

// ---- y = add + the choices' parts, in the order of their keys; a thread owns 8 adjacent channels.  Bound by memory: 2048 tokens of 6
// choices, D 2048, 109 MB in 18 us, most of it out of the memory-side cache.
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
    const int32_t* ids = a.ids + (int64_t)t * a.k;
    const float* part = a.part + (int64_t)t * a.k * a.D + c;
    for (int j0 = 0; j0 < a.k; j0 += 4) {                        // (four at once; the part of a choice that is left out holds anything)
        f32x4 p[4][2];
        int id[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = min(j0 + i, a.k - 1);
            p[i][0] = reinterpret_cast<const f32x4*>(part + (int64_t)j * a.D)[0];
            p[i][1] = reinterpret_cast<const f32x4*>(part + (int64_t)j * a.D)[1];
            id[i] = j0 + i < a.k ? ids[j] : -1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (id[i] >= 0)
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] += p[i][q / 4][q % 4];
    }
    bf16x8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (__bf16)v[q];
    *reinterpret_cast<bf16x8*>(a.y + (int64_t)t * a.ldy + c) = o;
}

// ---- A few tokens: the choice with the first product, the second one with the sum, in two launches behind the router's sums, by the waves and rings of
// gdn_few_kernel.h.  P > 0: every workgroup of a token chooses anew; P = 0: the choices have been made.
template <typename C, int P>
__global__ void __launch_bounds__(64 * C::WAVES) moe_up_few_kernel(MoeArgs a) {          // WR / 2 of a choice's F; grid: (2 F / WR, T k)
    extern __shared__ __align__(16) char smem[];
    __shared__ int32_t chosen;
    __shared__ float weight;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pair = blockIdx.y, t = pair / a.k, j = pair % a.k, f0 = blockIdx.x * (C::WR / 2);
    if constexpr (P > 0) {
        if (wave == 0) {
            int id;
            float p;
            choose<P>(a, t, lane, id, p);
            if (lane == j) { chosen = p != 0.f ? id : -1; weight = p; }
            if (lane < a.k && j == 0 && blockIdx.x == 0) {
                if (a.out_ids) a.out_ids[pair + lane] = id;
                if (a.out_weights) a.out_weights[pair + lane] = p;
                a.ids[pair + lane] = p != 0.f ? id : -1;
            }
        }
        __syncthreads();
    }
    const int e = __builtin_amdgcn_readfirstlane(P > 0 ? chosen : a.ids[pair]);
    if (e < 0) return;
    const int bytes = C::WR / 2 * a.D * 2;
    const few::Part gate = {reinterpret_cast<const char*>(a.w_gate_up + ((int64_t)e * 2 * a.F + f0) * a.D), bytes, a.D * 2};
    const few::Part up = {gate.at + (int64_t)a.F * a.D * 2, bytes, a.D * 2};
    const few::Part x = {reinterpret_cast<const char*>(a.x + t * a.ldx), a.D * 2, a.D * 2};      // one row: the others of its tile are behind its end, zeros
    f32x4 acc[C::CT];
#pragma unroll
    for (int i = 0; i < C::CT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (where k begins, see gdn_linear_few_kernel: by the expert and its rows, not by the choice's place in the batch, so that a row's sums are the same wherever its token stands)
    const int steps = a.D / few::STEP, first = (int)((blockIdx.x + 3u * (uint32_t)e) * 5u % (uint32_t)steps);
    C::sums_of(acc, gate, up, x, steps,
                   [&](int step, few::Part&, few::Part&, few::Part&) { return (step + first >= steps ? step + first - steps : step + first) * few::STEP * 2; },
                   smem + wave * C::RING, wave, lane);
    __builtin_amdgcn_s_waitcnt(0x0F70);                          // (no load of an empty descriptor writes behind the sums)
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    C::put_sums(acc, sums, wave, lane);
    __syncthreads();
    if (threadIdx.x < C::WR / 8) {
        const int piece = threadIdx.x;
        const f32x4 v = (P > 0 ? weight : a.weights[pair]) * (activate(a.act, C::get_sum(sums, 0, piece)) * C::get_sum(sums, 0, piece + C::WR / 8));
        // (rounded to bf16 as in the tiles, whose second product takes it so: a token's row does not change with how many stand beside it but for the order of fp32 sums)
        *reinterpret_cast<bf16x4*>(a.h + (int64_t)pair * a.F + f0 + 4 * piece) = __builtin_convertvector(v, bf16x4);
    }
}

template <typename C>
__global__ void __launch_bounds__(64 * C::WAVES) moe_down_few_kernel(MoeArgs a) {        // WR of a token's D; grid: (D / WR, T)
    extern __shared__ __align__(16) char smem[];
    __shared__ int32_t ids[MAX_K], at[MAX_K];                    // the choices that count, and which they are
    __shared__ int32_t count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.y, d0 = blockIdx.x * C::WR;
    if (wave == 0) {
        const int id = lane < a.k ? a.ids[t * a.k + lane] : -1;
        const uint64_t in = __ballot(id >= 0);
        if (id >= 0) {
            const int n = __popcll(in & ((1ull << lane) - 1));
            ids[n] = id;
            at[n] = lane;
        }
        if (lane == 0) count = __popcll(in);
    }
    __syncthreads();
    const int per = a.F / few::STEP, n = __builtin_amdgcn_readfirstlane(count), steps = n * per;
    const int my_id = lane < n ? ids[lane] : 0, my_at = lane < n ? at[lane] : 0;      // (in a lane each: a read of LDS would wait for the loads to LDS)
    const int64_t expert = (int64_t)a.D * a.F * 2;
    const few::Part w0 = {reinterpret_cast<const char*>(a.w_down + (int64_t)d0 * a.F), C::WR * a.F * 2, a.F * 2};
    const few::Part w1 = {w0.at + (int64_t)8 * C::HALF * a.F * 2, w0.bytes - 8 * C::HALF * a.F * 2, a.F * 2};
    const few::Part x = {reinterpret_cast<const char*>(a.h + (int64_t)t * a.k * a.F), a.F * 2, a.F * 2};
    f32x4 acc[C::CT];
#pragma unroll
    for (int i = 0; i < C::CT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int first = steps ? (int)(blockIdx.x * 5u % (uint32_t)steps) : 0;
    C::sums_of(acc, w0, w1, x, steps,
               [&](int step, few::Part& v0, few::Part& v1, few::Part& vx) {
                   const int s = step + first >= steps ? step + first - steps : step + first, j = s / per;
                   const int64_t skip = from_lane(my_id, j) * expert;
                   v0.at += skip;
                   v1.at += skip;
                   vx.at += (int64_t)from_lane(my_at, j) * a.F * 2;
                   return (s - j * per) * few::STEP * 2;
               },
               smem + wave * C::RING, wave, lane);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    C::put_sums(acc, sums, wave, lane);
    __syncthreads();
    if (threadIdx.x < C::WR / 4) {
        const int d = d0 + 4 * threadIdx.x;
        f32x4 v = C::get_sum(sums, 0, threadIdx.x);
        if (a.add) v += __builtin_convertvector(*reinterpret_cast<const bf16x4*>(a.add + t * a.ld_add + d), f32x4);
        *reinterpret_cast<bf16x4*>(a.y + t * a.ldy + d) = __builtin_convertvector(v, bf16x4);
    }
}

}  // namespace moe
}  // namespace gdn
