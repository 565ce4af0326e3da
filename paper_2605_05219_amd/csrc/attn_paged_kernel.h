// Device side of the paged cache's own operators (see include/attn_paged.h): rotary positions with the append, the attention weight
// that cached rows gather, and eviction by it.  The attention over the pages is attn_kernel.h's, with PagedArgs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_kernel.h"

namespace attn {

// A call's index arrays ("plan"): in device memory, or by value in the arguments of its launches where they are few words, which spares the
// launch that would write them there (one token 10.4 against 12.7 us, an eviction of 8200 rows 20.3 against 22.4).
template <bool BY_VALUE>
struct PlanWords {
    int32_t w[BY_VALUE ? PLAN_WORDS : 1];
};

// The request with cu[r] <= t < cu[r + 1], for a wave: 64 of the ends at a time, one in each lane.
__device__ __forceinline__ int request_of(const int32_t* cu, int n_req, int t) {
    const int lane = threadIdx.x & 63;
    int r = 0;
    for (int base = 0; base < n_req; base += 64) {
        const int n = __popcll(__ballot(base + lane < n_req && cu[base + lane + 1] <= t));
        r += n;
        if (n < 64) break;
    }
    return r;
}

// ---------------------------------------------------------------- rotary positions and the append
// A position's angle in turns is position * turns-per-position modulo 1: with the latter as a 64-bit fraction the product wraps
// exactly, so that far positions keep 2^-32 of a turn.
constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TOKENS = 8;        // tokens per workgroup, at most
constexpr int ROPE_UNITS = 4;         // pieces of 16 elements that a thread has on their way at once

struct RopeArgs {
    const void *q, *k, *v;
    uint16_t* q_out;
    uint16_t *k_pool, *v_pool;
    const int32_t* plan;              // cu (n_req + 1), start, pos, place (n_req each: where the page of row 0 would be listed), page ids
    int64_t ldq, ldk, ldv, page_stride;
    int32_t n_req, T, tokens;         // tokens: per workgroup
    int32_t H_q, H_kv, unit_shift;    // log2 of the pieces of 16 elements per head, d / 16
    int32_t page_shift, rot, layout;
    float amplitude;
    uint64_t turn[128];               // turns per position, 2^-64
};

// Eight elements as they come (two or one 16-byte loads), and as floats.
template <bool F32>
struct Raw8 {
    u32x4 r[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        if constexpr (F32) {
            const u32x4* const s = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + at);
            r[0] = s[0];
            r[1] = s[1];
        } else {
            r[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
        }
    }
    __device__ __forceinline__ void floats(float* x) const {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t u = r[i / 4][i % 4];           // (a value: a cast of the vector's element itself takes the first)
                x[i] = __builtin_bit_cast(float, u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __builtin_bit_cast(float, r[0][i] << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, r[0][i] & 0xffff0000u);
            }
        }
    }
};
__device__ __forceinline__ void store8_bf16(uint16_t* p, const float* x) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)x[i];
    *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, y);
}
__device__ __forceinline__ void store8_fp16(uint16_t* p, const float* x) {
    half8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (_Float16)x[i];
    *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, y);
}

// One workgroup takes `tokens` tokens: one thread per 16 elements of a head (two runs of 8), ROPE_UNITS of them on
// their way while the tokens' places in the pages are looked up and their cosines and sines made, once for all heads, in LDS.
// Bound: memory, read and written once: 352 MB (fp32 in, 16 heads of 256 and 4) in 71 us, 4.9 TB/s; 84 MB (a prompt of 8192 tokens) in 18.5 us, of which
// 5 are its one round's start.
template <bool F32, bool BY_VALUE>
__global__ void __launch_bounds__(ROPE_THREADS) attn_rope_kernel(RopeArgs a, PlanWords<BY_VALUE> words) {
    __shared__ float cs[ROPE_TOKENS][2][128];
    __shared__ int64_t row_at[ROPE_TOKENS];      // the token's row in the pools, head 0
    __shared__ int32_t position[ROPE_TOKENS];
    const int tok0 = (int)blockIdx.x * a.tokens;
    const int n_tok = min(a.tokens, a.T - tok0);
    const int tid = threadIdx.x, wave = tid >> 6;
    const int D = 16 << a.unit_shift, half = a.rot >> 1;
    const int per = (a.H_q + 2 * a.H_kv) << a.unit_shift, total = n_tok * per;
    const int step_t = ROPE_THREADS / per, step_j = ROPE_THREADS - step_t * per;

    Raw8<F32> raw[ROPE_UNITS][2];
    int next_t = tid / per, next_j = tid - next_t * per;      // the unit to be loaded: its token, its number among the token's
    // a unit's places: elements lo .. lo + 7 and hi .. hi + 7 of its head, of the first and the second half of the part that turns, of the part that
    // does not, or of a value (so that neighbouring threads load and store neighbouring 16 bytes)
    auto runs_of = [&](int j, int& head, int& lo, int& hi, bool& turned) __attribute__((always_inline)) {
        head = j >> a.unit_shift;
        const int u = j & ((1 << a.unit_shift) - 1), rot = head < a.H_q + a.H_kv ? a.rot : 0;
        turned = 16 * u < rot;
        lo = turned ? 8 * u : rot + 8 * u - (rot >> 1);
        hi = lo + (turned ? half : (D - rot) >> 1);
    };
    auto on = [&](int& t, int& j) __attribute__((always_inline)) {
        t += step_t;
        j += step_j;
        if (j >= per) { j -= per; ++t; }
    };
    auto load_units = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ROPE_UNITS; ++i) {
            if (next_t < n_tok) {
                int head, lo, hi;
                bool turned;
                runs_of(next_j, head, lo, hi, turned);
                const int64_t tok = tok0 + next_t;
                const bool is_q = head < a.H_q, is_k = head < a.H_q + a.H_kv;
                const void* const from = is_q ? a.q : is_k ? a.k : a.v;
                const int64_t at = tok * (is_q ? a.ldq : is_k ? a.ldk : a.ldv) + (head - (is_q ? 0 : is_k ? a.H_q : a.H_q + a.H_kv)) * D;
                raw[i][0].load(from, at + lo);
                raw[i][1].load(from, at + hi);
            }
            on(next_t, next_j);
        }
    };
    int t = next_t, j = next_j;                               // the unit to be stored
    load_units();

    const int32_t* const cu = BY_VALUE ? words.w : a.plan;
    const int32_t *const start = cu + a.n_req + 1, *const pos = start + a.n_req, *const place = pos + a.n_req, *const page_ids = place + a.n_req;
    for (int i = wave; i < n_tok; i += ROPE_THREADS / 64) {
        const int r = request_of(cu, a.n_req, tok0 + i);
        if ((tid & 63) == 0) {
            const int in = tok0 + i - cu[r], row = start[r] + in;
            position[i] = pos[r] + in;
            row_at[i] = (int64_t)page_ids[place[r] + (row >> a.page_shift)] * a.page_stride + (int64_t)(row & ((1 << a.page_shift) - 1)) * D;
        }
    }
    __syncthreads();
    for (int i = tid; i < n_tok * half; i += ROPE_THREADS) {
        const int tk = i / half, p = i - tk * half;
        const uint64_t turns = (uint64_t)(uint32_t)position[tk] * a.turn[p];
        float sn, cn;
        sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &sn, &cn);
        cs[tk][0][p] = cn * a.amplitude;
        cs[tk][1][p] = sn * a.amplitude;
    }
    __syncthreads();
    for (int done = 0; done < total; done += ROPE_THREADS * ROPE_UNITS) {
        if (done > 0) load_units();
#pragma unroll
        for (int i = 0; i < ROPE_UNITS; ++i) {
            if (t < n_tok) {
                int head, lo, hi;
                bool turned;
                runs_of(j, head, lo, hi, turned);
                float x[16];
                raw[i][0].floats(x);
                raw[i][1].floats(x + 8);
                if (head >= a.H_q + a.H_kv) {                 // a value: widened
                    uint16_t* const dst = a.v_pool + row_at[t] + ((int64_t)(head - a.H_q - a.H_kv) * D << a.page_shift) + lo;
                    store8_fp16(dst, x);
                    store8_fp16(dst + hi - lo, x + 8);
                } else {
                    if (turned) {
                        const float *const c = cs[t][0], *const s = cs[t][1];
                        float y[16];
                        if (a.layout == 0) {                  // pair lo + e: its halves are e of the two runs
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                y[e] = x[e] * c[lo + e] - x[8 + e] * s[lo + e];
                                y[8 + e] = x[8 + e] * c[lo + e] + x[e] * s[lo + e];
                            }
                        } else {                              // four pairs in each run
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int p = (e < 4 ? lo : hi) / 2 + (e & 3);
                                y[2 * e] = x[2 * e] * c[p] - x[2 * e + 1] * s[p];
                                y[2 * e + 1] = x[2 * e + 1] * c[p] + x[2 * e] * s[p];
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = y[e];
                    }
                    uint16_t* const dst = head < a.H_q ? a.q_out + ((int64_t)(tok0 + t) * a.H_q + head) * D
                                                       : a.k_pool + row_at[t] + ((int64_t)(head - a.H_q) * D << a.page_shift);
                    store8_bf16(dst + lo, x);
                    store8_bf16(dst + hi, x + 8);
                }
            }
            on(t, j);
        }
    }
}

// ---------------------------------------------------------------- the weight that cached rows gather
// A key's sum runs over query rows, so keys stay and queries pass: each of the four waves of a workgroup holds 64 keys (32 at d = 256; at d = 64 there are eight
// waves with 32 each, 8192 tokens of 16 heads 126 -> 117 us, which at d = 128 gains 2 % or loses 3) in registers as matrix operands, tiles of 64 query rows (tokens x heads of the group, row = token * G + head) go through two LDS stages, brought by loads to LDS a
// tile ahead.  S[row][key] puts a key into a lane's column and 16 of 32 rows into its registers: the sum over rows needs no
// exchange between lanes but one with the other half at the end, and no atomics.  A row's log-sum-exp comes by LDS in units of log2.
// Bound: matrix and vector units alike (8192 tokens of 16 heads, d = 128: 55 us of products and 70 us of multiply-adds, exponentials and
// sums at 2.4 GHz), so a wave computes the products of the next 32 rows in between the exponentials of the last (in turn they took 40 % more).  The call takes
// 157 to 163 us by card (875 TFLOP/s): matrix units busy 0.40, vector units 0.50 of 341 k clocks at a power-limited 2.1 GHz, two waves to a SIMD (registers); a unit's
// start (4 us, three rounds) and the last round cost 25 of them.  500 tokens behind 7700 rows, d = 64: 24 us.
constexpr int WGT_THREADS = 256;      // of the few-rows kernel
__host__ __device__ constexpr int wgt_waves(int d) { return d == 64 ? 8 : 4; }
__host__ __device__ constexpr int wgt_keys(int d) { return d == 256 ? 128 : 256; }   // keys per workgroup
constexpr int WGT_ROWS = 64;          // query rows per tile
constexpr int WGT_PARTS = 16384;      // partial sums (of a tile of keys, a part of its rows, a head) of a call, at most
constexpr int WGT_FEW = 16;           // rows of a request of the few-rows kernel, at most
constexpr int WGT_REC = 8;            // a unit's record: first token, tokens, start, place, first key, first row, one past the last, partial sum or -1
constexpr int WGT_MERGE = 5;          // a cut tile's record: tokens + start, start, place, first key, first partial sum; one past the last is the next one's

struct WeightArgs {
    const uint16_t* q;
    const float* lse;
    const uint16_t* k_pool;
    const float* w_in;        // or nullptr
    float* w_out;
    const int32_t* plan;      // WGT_REC ints per unit of either kernel, WGT_MERGE per tile whose rows are cut (and the first partial sum behind the last one), page ids
    int32_t units, merges, ids;   // where each begins (units: of the kernel launched)
    float* part;              // [partial sum][head][keys of a tile]
    int64_t page_stride, w_stride;
    int32_t H_q, H_kv, G;
    int32_t page_shift;
    float inv_G;              // 1 / G: x / G = (int)((x + 1/2) inv_G) for the small x that it is used for
    float scale_log2e, decay;
};

template <int D>
struct WeightSmem {
    static constexpr int CPR = D / 8, ROW_BYTES = D * 2, TILE_BYTES = WGT_ROWS * ROW_BYTES;
    static constexpr int PPW = TILE_BYTES / (1024 * wgt_waves(D));       // 1 KiB loads per wave and tile
    static __device__ __forceinline__ int f(int row) { return CPR >= 16 ? (row & 15) : ((row >> 1) & 7); }
};

__device__ __forceinline__ void store_weight(const WeightArgs& a, const int32_t* page_ids, int place, int kvh, int c0, int key, float sum) {
    const int64_t at = (int64_t)page_ids[place + (key >> a.page_shift)] * a.w_stride + ((int64_t)kvh << a.page_shift) + (key & ((1 << a.page_shift) - 1));
    a.w_out[at] = (a.w_in && key < c0 ? a.decay * a.w_in[at] : 0.f) + sum;
}

template <int D, bool BY_VALUE>
__global__ void __launch_bounds__(64 * wgt_waves(D), wgt_waves(D) / 2) attn_weights_kernel(WeightArgs a, PlanWords<BY_VALUE> words) {
    typedef WeightSmem<D> SM;
    constexpr int KB = D / 16, KEYS = wgt_keys(D), NB = KEYS / (32 * wgt_waves(D));      // NB: blocks of 32 keys per wave
    constexpr int AHEAD_TILES = D == 256 ? 1 : 2;    // a tile is asked for this many tiles ahead (three stages at d = 256 would leave one workgroup to a compute unit)
    __shared__ __attribute__((aligned(1024))) char stage0[SM::TILE_BYTES], stage1[SM::TILE_BYTES], stage2[AHEAD_TILES == 2 ? SM::TILE_BYTES : 16];
    __shared__ __attribute__((aligned(16))) float neg_lse[4][WGT_ROWS];   // -lse log2(e); rows past the end -inf
    __shared__ __attribute__((aligned(16))) int limit[4][WGT_ROWS];       // last key a row sees; rows past the end -1

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, g = lane >> 5;
    const int kvh = (int)blockIdx.x % a.H_kv;
    const int32_t *const plan = BY_VALUE ? words.w : a.plan, *const page_ids = plan + a.ids;
    const int32_t* const rec = plan + a.units + (int64_t)((int)blockIdx.x / a.H_kv) * WGT_REC;
    const int tok0 = rec[0], n = rec[1], c0 = rec[2], place = rec[3], kv0 = rec[4], row_lo = rec[5], row_hi = rec[6], part = rec[7];
    const int kv_len = c0 + n;

    // ---- this wave's keys: operand B, column = key, d = 16 kb + 8 g + {0..7}
    const int key0 = kv0 + 32 * NB * wave;
    int page[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) page[b] = page_ids[place + (min(key0 + 32 * b + col, kv_len - 1) >> a.page_shift)];

    // ---- the next tile to bring: its first row, that row's token and head (uniform; a tile is step_t tokens and step_h heads on)
    const int step_t = WGT_ROWS / a.G, step_h = WGT_ROWS - step_t * a.G;
    int row_n = row_lo, t_n = row_lo / a.G, h_n = row_lo - t_n * a.G;
    const int64_t tok_bytes = (int64_t)a.H_q * D * 2;
    const float* const lse_base = a.lse + (int64_t)tok0 * a.H_q + kvh * a.G;
    const uint16_t* const q_base = a.q + ((int64_t)tok0 * a.H_q + kvh * a.G) * D;
    // where a lane's 16-byte chunks of a tile and its row's sum lie from the tile's first token: the same for every tile where tiles begin with a token's
    // first head (64 a multiple of G)
    int voff[SM::PPW], lse_t = 0, lse_off = 0;
    auto places = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SM::PPW; ++i) {
            const int s = (wave * SM::PPW + i) * 64 + lane, rr = s / SM::CPR, pos = s % SM::CPR;
            const int x = h_n + rr, t = (int)(((float)x + 0.5f) * a.inv_G);
            voff[i] = (t * a.H_q + x - t * a.G) * D * 2 + ((pos ^ SM::f(rr)) << 4);
        }
        const int x = h_n + ((int)threadIdx.x & (WGT_ROWS - 1));
        lse_t = (int)(((float)x + 0.5f) * a.inv_G);
        lse_off = lse_t * a.H_q + x - lse_t * a.G;
    };
    places();
    float lse_n = 0.f;           // of row row_n + thread (the first 64 threads)
    int lim_n = 0;
    // to LDS, 16-byte chunk c of a row at c ^ f(row); rows past the request's last one come as zeros
    auto issue = [&](char* sb) __attribute__((always_inline)) {
        if (step_h != 0) places();
        if (threadIdx.x < WGT_ROWS) {
            const bool row = row_n + (int)threadIdx.x < row_hi;
            lim_n = row ? c0 + t_n + lse_t : -1;
            lse_n = row ? lse_base[(int64_t)t_n * a.H_q + lse_off] : INFINITY;
        }
        const uint16_t* const base = q_base + (int64_t)t_n * (a.H_q * D);
        const int bytes = (int)min((int64_t)INT32_MAX, (int64_t)(n - 1 - t_n) * tok_bytes + a.G * D * 2);
#pragma unroll
        for (int i = 0; i < SM::PPW; ++i) load_to_lds(base, bytes, sb + (wave * SM::PPW + i) * 1024, voff[i], 0);
        row_n += WGT_ROWS;
        t_n += step_t;
        h_n += step_h;
        if (h_n >= a.G) { h_n -= a.G; ++t_n; }
    };
    auto stage_rows = [&](int st, float lse, int lim) __attribute__((always_inline)) {    // what issue() fetched of the rows' sums goes to LDS
        if (threadIdx.x < WGT_ROWS) {
            neg_lse[st][threadIdx.x] = -lse * 1.4426950408889634f;
            limit[st][threadIdx.x] = lim;
        }
    };
    // the first tiles are on their way while the page ids come, behind which the keys can be asked for
    const bool any = row_lo < row_hi, second = AHEAD_TILES == 2 && row_lo + WGT_ROWS < row_hi;
    float lse0 = 0.f;
    int lim0 = 0;
    if (any) {
        issue(stage0);
        lse0 = lse_n;
        lim0 = lim_n;
        if (second) issue(stage1);
    }
    bf16x8 kf[NB][KB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int key = min(key0 + 32 * b + col, kv_len - 1);
        const uint16_t* const kp = a.k_pool + (int64_t)page[b] * a.page_stride + ((int64_t)kvh * D << a.page_shift) +
                                   (int64_t)(key & ((1 << a.page_shift) - 1)) * D + 8 * g;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) kf[b][kb] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(kp + 16 * kb));
    }
    float acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = 0.f;
    // the logits of 32 rows of a stage
    auto products = [&](f32x16 (&S)[NB], const char* sb, int sub) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[b][i] = 0.f;
        const char* const qrow = sb + (32 * sub + col) * SM::ROW_BYTES;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const bf16x8 qf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + (((2 * kb + g) ^ SM::f(col)) << 4)));
#pragma unroll
            for (int b = 0; b < NB; ++b) S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[b][kb], S[b], 0, 0, 0);
        }
    };
    // the weights of 32 rows, summed, four of a block (registers 4 q .. 4 q + 3) at a time; CUT: some row does not see some key of this wave, or is past
    // the last one (whose zeros an infinite key turns into what is not a number)
    auto sum4 = [&](const f32x16& S, int b, int q, f32x4 nl, const int* lim, auto cut) __attribute__((always_inline)) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[4 * q + e], a.scale_log2e, nl[e]));
            if constexpr (decltype(cut)::value)
                if (key0 + 32 * b + col > lim[e]) p[e] = 0.f;
        }
        acc[b] += (p[0] + p[1]) + (p[2] + p[3]);
    };
    auto sums = [&](const f32x16 (&S)[NB], int st, int sub) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at = 32 * sub + 8 * q + 4 * g;
#pragma unroll
            for (int b = 0; b < NB; ++b) sum4(S[b], b, q, *reinterpret_cast<const f32x4*>(&neg_lse[st][at]), &limit[st][at], std::true_type{});
        }
    };
    // both, of different rows, in turn: the products of a step of the contraction, then the vector work of four weights or more, which the
    // products in flight cover; nothing moves from step to step
    auto both_cut = [&](f32x16 (&Sn)[NB], const char* sb, int sub_n, const f32x16 (&Sp)[NB], int st, int sub_p, auto cut) __attribute__((always_inline)) {
        constexpr int AHEAD = 3;                         // operand fragments read ahead
        constexpr int LATE = KB >= 8 ? KB / 4 : 1;       // steps before the first weights: the last products of these and their rows' sums are on their way
        const char* const qrow = sb + (32 * sub_n + col) * SM::ROW_BYTES;
        auto fragment = [&](int kb) __attribute__((always_inline)) { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + (((2 * kb + g) ^ SM::f(col)) << 4))); };
        bf16x8 qf[KB];
        f32x4 nl[4];
#pragma unroll
        for (int kb = 0; kb < AHEAD; ++kb) qf[kb] = fragment(kb);
#pragma unroll
        for (int q = 0; q < 4; ++q) nl[q] = *reinterpret_cast<const f32x4*>(&neg_lse[st][32 * sub_p + 8 * q + 4 * g]);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) Sn[b][i] = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            __builtin_amdgcn_sched_barrier(0);
            if (kb + AHEAD < KB) qf[kb + AHEAD] = fragment(kb + AHEAD);
#pragma unroll
            for (int b = 0; b < NB; ++b) Sn[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[kb], kf[b][kb], Sn[b], 0, 0, 0);
#pragma unroll
            for (int x = 4 * NB * max(kb - LATE, 0) / (KB - LATE); x < 4 * NB * max(kb + 1 - LATE, 0) / (KB - LATE); ++x)
                sum4(Sp[x % NB], x % NB, x / NB, nl[x / NB], &limit[st][32 * sub_p + 8 * (x / NB) + 4 * g], cut);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto both = [&](f32x16 (&Sn)[NB], const char* sb, int sub_n, const f32x16 (&Sp)[NB], int st, int sub_p, bool cut) __attribute__((always_inline)) {
        if (cut) both_cut(Sn, sb, sub_n, Sp, st, sub_p, std::true_type{});
        else both_cut(Sn, sb, sub_n, Sp, st, sub_p, std::false_type{});
    };
    // Tile i has its rows' sums in slot i & 3 (a wave may still be at the last rows of tile i - 1 when another stages those of the tile ahead).
    f32x16 A[NB], B[NB];
    if (any) {
        int row = row_lo, i = 0;
        const int cut_end = max(key0 + 32 * NB - 1 - c0, 0) * a.G;      // rows before it do not see all of this wave's keys
        stage_rows(0, lse0, lim0);
        if (second) stage_rows(1, lse_n, lim_n);
        wait_vmcnt<0>();
        __syncthreads();
        products(A, stage0, 0);
        // a tile from its second half to the first half of the next; `ahead`: the stage that the tile before left.  False: it was the last one.
        auto step = [&](const char* sb, const char* next, char* ahead) __attribute__((always_inline)) {
            const bool more = row + AHEAD_TILES * WGT_ROWS < row_hi, cut = row < cut_end || row + WGT_ROWS > row_hi;
            if (more) issue(ahead);
            both(B, sb, 1, A, i & 3, 0, cut);
            if (row + WGT_ROWS >= row_hi) return false;
            if (more) {
                stage_rows((i + AHEAD_TILES) & 3, lse_n, lim_n);
                wait_vmcnt<AHEAD_TILES == 2 ? SM::PPW : 0>();
            } else {
                wait_vmcnt<0>();
            }
            __syncthreads();
            both(A, next, 0, B, i & 3, 1, cut);
            row += WGT_ROWS;
            ++i;
            return true;
        };
        for (;;) {
            if constexpr (AHEAD_TILES == 2) {
                if (!step(stage0, stage1, stage2) || !step(stage1, stage2, stage0) || !step(stage2, stage0, stage1)) break;
            } else {
                if (!step(stage0, stage1, stage1) || !step(stage1, stage0, stage0)) break;
            }
        }
        sums(B, i & 3, 1);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float sum = sum_with_other_half(acc[b]);
        const int key = key0 + 32 * b + col;
        if (g != 0 || key >= kv_len) continue;
        if (part < 0) store_weight(a, page_ids, place, kvh, c0, key, sum);
        else a.part[((int64_t)part * a.H_kv + kvh) * KEYS + key - kv0] = sum;
    }
}

// The same for requests of at most 16 rows (decoding): bound by the keys' bytes, so that nothing is shared between waves and none waits for
// another.  A wave holds 64 keys as four blocks of columns of 16x16x32 products, 64 contiguous bytes of a key per load and lane group, all of them in
// flight at once, four workgroups to a compute unit; the query rows come straight from memory.  64 requests behind 4 to 10 thousand rows, 233 MB: 47 us, 4.9
// TB/s (68 by the kernel above; the same when a workgroup walks a run of tiles and asks for the next tile's keys as it goes).
template <int D, bool BY_VALUE>
__global__ void __launch_bounds__(WGT_THREADS, D == 256 ? 2 : 4) attn_weights_few_kernel(WeightArgs a, PlanWords<BY_VALUE> words) {
    constexpr int KS = D / 32, NB = wgt_keys(D) / 64;       // NB: blocks of 16 keys per wave
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i16 = lane & 15, g = lane >> 4;
    const int kvh = (int)blockIdx.x % a.H_kv;
    const int32_t *const plan = BY_VALUE ? words.w : a.plan, *const page_ids = plan + a.ids;
    const int32_t* const rec = plan + a.units + (int64_t)((int)blockIdx.x / a.H_kv) * WGT_REC;
    const int tok0 = rec[0], n = rec[1], c0 = rec[2], place = rec[3], rows = rec[6];
    const int kv_len = c0 + n, key0 = rec[4] + 16 * NB * wave;
    if (key0 >= kv_len) return;
    const int mask = (1 << a.page_shift) - 1;
    u32x4 kf[NB][KS];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int key = min(key0 + 16 * b + i16, kv_len - 1);
        const uint16_t* const kp = a.k_pool + (int64_t)page_ids[place + (key >> a.page_shift)] * a.page_stride + ((int64_t)kvh * D << a.page_shift) +
                                   (int64_t)(key & mask) * D + 8 * g;
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[b][s] = *reinterpret_cast<const u32x4*>(kp + 32 * s);
    }
    // the key whose sum this lane stores
    const int mine = key0 + lane;
    const bool stores = lane < 16 * NB && mine < kv_len;
    int64_t at = 0;
    float held = 0.f;
    if (stores) {
        at = (int64_t)page_ids[place + (mine >> a.page_shift)] * a.w_stride + ((int64_t)kvh << a.page_shift) + (mine & mask);
        if (a.w_in && mine < c0) held = a.w_in[at];
    }
    // query rows: operand A, row i16, d = 32 s + 8 g + {0..7};  the sums: rows 4 g + e
    bf16x8 qf[KS];
    float nl[4];
    int lim[4];
    {
        const int row = min(i16, rows - 1), t = row / a.G;
        const uint16_t* const qp = a.q + ((int64_t)(tok0 + t) * a.H_q + kvh * a.G + row - t * a.G) * D + 8 * g;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 32 * s));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int x = 4 * g + e, te = min(x, rows - 1) / a.G;
            lim[e] = x < rows ? c0 + te : -1;
            nl[e] = -a.lse[(int64_t)(tok0 + te) * a.H_q + kvh * a.G + min(x, rows - 1) - te * a.G] * 1.4426950408889634f;
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[s], __builtin_bit_cast(bf16x8, kf[b][s]), S, 0, 0, 0);
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[e], a.scale_log2e, nl[e]));
            if (key0 + 16 * b + i16 > lim[e]) p[e] = 0.f;
        }
        const float all = sum_over_groups((p[0] + p[1]) + (p[2] + p[3]));
        if (g == b) sum = all;
    }
    if (stores) a.w_out[at] = (a.w_in && mine < c0 ? a.decay * held : 0.f) + sum;
}

// The parts of a tile's rows, summed in order; one workgroup per (tile, head) and one thread per key.
template <int KEYS, bool BY_VALUE>
__global__ void __launch_bounds__(KEYS) attn_weights_merge_kernel(WeightArgs a, PlanWords<BY_VALUE> words) {
    const int kvh = (int)blockIdx.x % a.H_kv;
    const int32_t *const plan = BY_VALUE ? words.w : a.plan, *const page_ids = plan + a.ids;
    const int32_t* const rec = plan + a.merges + (int64_t)((int)blockIdx.x / a.H_kv) * WGT_MERGE;
    const int kv_len = rec[0], c0 = rec[1], place = rec[2], kv0 = rec[3], p0 = rec[4], p1 = rec[WGT_MERGE + 4];
    const int key = kv0 + (int)threadIdx.x;
    if (key >= kv_len) return;
    float sum = 0.f;
#pragma unroll 8
    for (int p = p0; p < p1; ++p) sum += a.part[((int64_t)p * a.H_kv + kvh) * KEYS + threadIdx.x];
    store_weight(a, page_ids, place, kvh, c0, key, sum);
}

// ---------------------------------------------------------------- eviction
struct EvictArgs {
    uint16_t *k_pool, *v_pool;
    float* w_pool;
    int32_t* index;
    const int32_t* plan;
    int64_t page_stride, w_stride;
    int32_t n_req, H_kv, page_shift;
};

// The arrays of an eviction's plan.
struct EvictPlan {
    const int32_t *rows, *keep, *first, *recent;          // keep: at most rows
    const int32_t *place, *new_place;                     // where a request's old and new pages begin in page_ids
    const int32_t *keep_cu, *block_cu;                    // n_req + 1: kept rows, and workgroups of the copy for one head, before each request
    const int32_t* page_ids;
    __host__ __device__ EvictPlan(const int32_t* p, int64_t n)
        : rows(p), keep(p + n), first(p + 2 * n), recent(p + 3 * n), place(p + 4 * n), new_place(p + 5 * n), keep_cu(p + 6 * n),
          block_cu(p + 7 * n + 1), page_ids(p + 8 * n + 2) {}
};

// A weight's rank as an unsigned number: larger weights larger, -0 as +0, what is not a number 0.
__device__ __forceinline__ uint32_t weight_rank(float w) {
    if (w != w) return 0u;
    const uint32_t u = __builtin_bit_cast(uint32_t, w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over this lane and those before it, by lane exchanges inside the vector unit (within rows of 16, then a row's last lane to the next rows).
__device__ __forceinline__ int wave_sum_upto(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // 1, 2, 4, 8 lanes down the row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // last lane of rows 0, 2 to rows 1, 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // last lane of row 1 to rows 2, 3
    return x;
}

// The rows that one (request, head) keeps, by one workgroup.  Of every 8192 rows a thread has eight, 1024 apart; the ranks of the first SEL_HELD blocks of
// 8192 stay in registers, those behind them are read again where they are needed.  One pass counts the ranks' highest 11 bits; the digit in
// which the smallest rank kept lies leaves few rows as a rule, one to a thread from there on; the next 11 bits are counted until one row or all bits are
// left.  The counts of every 64 rows, summed, then say where each one's rows go.
// Bound: latencies, and the instructions of one compute unit per head (four copies of the counters, because neighbouring weights share their
// highest bits).  8200 rows 15.7 us, 30000 rows 30 (four rounds of 8 bits over memory 24 and 91).  Behind 32768 rows each pass reads again what is not
// held: a call that keeps 2000 rows of two heads takes 33 us from 32768, 41 from 40000, 101 from 100000 and 188 from 200000.
constexpr int SEL_THREADS = 1024;
constexpr int SEL_OWN = 8;             // rows of a thread in a block
constexpr int SEL_HELD = 4;
constexpr int SEL_BITS = 11;
constexpr int SEL_COPIES = 4;

template <bool BY_VALUE>
__global__ void __launch_bounds__(SEL_THREADS) attn_select_kernel(EvictArgs a, PlanWords<BY_VALUE> words) {
    constexpr int WAVES = SEL_THREADS / 64, BINS = 1 << SEL_BITS, BLOCK = SEL_THREADS * SEL_OWN;
    static_assert(BINS == 2 * SEL_THREADS && SEL_COPIES == 4, "a thread sums two digits, four copies in one read each");
    __shared__ __attribute__((aligned(16))) int hist[BINS * SEL_COPIES];
    __shared__ uint32_t few[SEL_THREADS];
    __shared__ __attribute__((aligned(16))) int part[2][SEL_OWN * WAVES];
    __shared__ int wave_a[WAVES], found[3], n_few;
    const EvictPlan e(BY_VALUE ? words.w : a.plan, a.n_req);
    const int r = (int)blockIdx.x / a.H_kv, kvh = (int)blockIdx.x % a.H_kv;
    const int rows = e.rows[r], keep = e.keep[r], first = e.first[r], last = rows - e.recent[r];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t* const out = a.index + (int64_t)a.H_kv * e.keep_cu[r] + (int64_t)kvh * keep;
    if (keep == rows) {
        for (int j = tid; j < rows; j += SEL_THREADS) out[j] = j;
        return;
    }
    const int32_t* const ids = e.page_ids + e.place[r];
    const float* const w = a.w_pool + ((int64_t)kvh << a.page_shift);
    const int mask = (1 << a.page_shift) - 1;
    const int want = keep - first - e.recent[r];          // rows to take from [first, last), fewer than there are
    auto load = [&](int base, uint32_t (&x)[SEL_OWN]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SEL_OWN; ++i) {
            const int j = min(base + SEL_THREADS * i + tid, rows - 1);
            x[i] = weight_rank(w[(int64_t)ids[j >> a.page_shift] * a.w_stride + (j & mask)]);
        }
    };
    uint32_t held[SEL_HELD][SEL_OWN] = {};
    // f(number, ranks) of every block of rows
    auto each_block = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < SEL_HELD; ++b)
            if (b * BLOCK < rows) f(b, held[b]);
#pragma unroll 1
        for (int b = SEL_HELD; b < (rows - 1) / BLOCK + 1; ++b) {
            uint32_t x[SEL_OWN];
            load(b * BLOCK, x);
            f(b, x);
        }
    };
    // f(rank) of this thread's rows in [first, last)
    auto each_row = [&](auto f) __attribute__((always_inline)) {
        each_block([&](int b, const uint32_t (&x)[SEL_OWN]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < SEL_OWN; ++i) {
                const int j = b * BLOCK + SEL_THREADS * i + tid;
                if (j >= first && j < last) f(x[i]);
            }
        });
    };
    uint32_t edge = 0xffffffffu;                          // the smallest rank kept
    int left = 0;                                         // how many rows of it
    if (want > 0) {
        auto clear = [&](int digits) __attribute__((always_inline)) {
            for (int i = tid; i < digits; i += SEL_THREADS) *reinterpret_cast<u32x4*>(&hist[SEL_COPIES * i]) = u32x4{0u, 0u, 0u, 0u};
        };
        clear(BINS);
        if (tid == 0) n_few = 0;
#pragma unroll
        for (int b = 0; b < SEL_HELD; ++b)
            if (b * BLOCK < rows) load(b * BLOCK, held[b]);
        __syncthreads();
        int bits = 32;                                    // bits of the edge that are not known yet
        bool one_each = false;                            // the rows that agree in the others are few: thread t has one, if t < count
        uint32_t mine = 0;
        int count = 0;
        left = want;
        edge = 0u;
        while (bits > 0) {
            const int shift = max(0, bits - SEL_BITS), digits = bits == 32 ? BINS : 1 << (bits - shift);
            auto add = [&](uint32_t x) __attribute__((always_inline)) {
                atomicAdd(&hist[SEL_COPIES * ((x >> shift) & (digits - 1)) + (lane & (SEL_COPIES - 1))], 1);
            };
            if (one_each) {
                if (tid < count) add(mine);
            } else {
                each_row([&](uint32_t x) __attribute__((always_inline)) {
                    if (bits == 32 || x >> bits == edge >> bits) add(x);
                });
            }
            bits = shift;
            __syncthreads();
            // from the largest digit down: thread t has digits - 1 - 2 t and the one below
            auto count_of = [&](int d) { const u32x4 n = *reinterpret_cast<const u32x4*>(&hist[SEL_COPIES * d]); return (int)((n[0] + n[1]) + (n[2] + n[3])); };
            const int d0 = digits - 1 - 2 * tid, n0 = d0 >= 0 ? count_of(d0) : 0, n1 = d0 >= 1 ? count_of(d0 - 1) : 0;
            const int upto = wave_sum_upto(n0 + n1);
            if (lane == 63) wave_a[wave] = upto;
            __syncthreads();
            int before = upto - n0 - n1;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                const int n = wave_a[i];                  // (all of them, whichever wave: the reads do not wait for each other)
                before += i < wave ? n : 0;
            }
            if (before < left && before + n0 >= left) { found[0] = d0; found[1] = left - before; found[2] = n0; }
            else if (before + n0 < left && before + n0 + n1 >= left) { found[0] = d0 - 1; found[1] = left - before - n0; found[2] = n1; }
            if (bits > 0) clear(1 << (bits - max(0, bits - SEL_BITS)));      // (everybody's digits have been read)
            __syncthreads();
            edge |= (uint32_t)found[0] << bits;
            left = found[1];
            if (bits == 0) break;
            const bool was = one_each;
            one_each = found[2] <= SEL_THREADS;
            if (one_each && !was) {                       // a row to a thread from here on
                count = found[2];
                each_row([&](uint32_t x) __attribute__((always_inline)) {
                    if (x >> bits == edge >> bits) few[atomicAdd(&n_few, 1)] = x;
                });
                __syncthreads();
                mine = tid < count ? few[tid] : 0u;
            } else if (one_each && found[2] == 1) {       // one is left: it is the edge
                __syncthreads();                          // (found has been read)
                if (tid < count && mine >> bits == edge >> bits) found[0] = (int)mine;
                __syncthreads();
                edge = (uint32_t)found[0];
                break;
            } else if (one_each && mine >> bits != edge >> bits) {
                count = 0;                                // this thread's row is out
            }
        }
    }
    // ---- the rows kept, in order
    int taken = 0, ties = 0;                              // rows above the edge or always kept, rows at the edge, of the blocks before
    each_block([&](int b, const uint32_t (&x)[SEL_OWN]) __attribute__((always_inline)) {
        const int j0 = b * BLOCK + tid;
        int* const sums = part[b & 1];                    // of row sixty-fours, in order: (i, wave)
        uint64_t take[SEL_OWN], tie[SEL_OWN];
#pragma unroll
        for (int i = 0; i < SEL_OWN; ++i) {
            const int j = j0 + SEL_THREADS * i;
            take[i] = tie[i] = 0;
            if (b * BLOCK + SEL_THREADS * i + 64 * wave < rows) {
                const bool mid = j >= first && j < last;
                take[i] = __ballot(j < rows && (!mid || x[i] > edge));
                tie[i] = __ballot(mid && x[i] == edge);
            }
            if (lane == 0) sums[WAVES * i + wave] = __popcll(take[i]) | __popcll(tie[i]) << 16;    // (both sums of a block are below 2^16)
        }
        __syncthreads();
        const int s0 = sums[2 * lane], s1 = sums[2 * lane + 1];
        const int upto = wave_sum_upto(s0 + s1), before = upto - s0 - s1;
        const uint64_t below = (1ull << lane) - 1;
#pragma unroll
        for (int i = 0; i < SEL_OWN; ++i) {
            const int q = WAVES * i + wave;
            const int ahead = __builtin_amdgcn_readlane(before, q / 2) + (q & 1 ? __builtin_amdgcn_readlane(s0, q / 2) : 0);
            const int tie_at = ties + (ahead >> 16), at = taken + (ahead & 0xffff) + min(tie_at, left);
            const int n_tie = max(0, left - tie_at), my_tie = __popcll(tie[i] & below);      // ties kept are the first
            if ((take[i] >> lane & 1) || ((tie[i] >> lane & 1) && my_tie < n_tie)) out[at + __popcll(take[i] & below) + min(my_tie, n_tie)] = j0 + SEL_THREADS * i;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        taken += all & 0xffff;
        ties += all >> 16;
    });
}

// The kept rows go to the new pages: a workgroup copies consecutive ones of a head, a 16-byte chunk of k and of v of GATHER_PASSES rows per thread, all
// loads ahead of the stores.  Bound: memory, 1.06 GB in 203 us (rows of 256 bytes with gaps between them; 2 or 8 rows per thread 236 and 240 us a call against
// 238, ordinary loads 246, ordinary stores 253: what is copied is not read again soon).
constexpr int GATHER_THREADS = 256, GATHER_PASSES = 4;
__host__ __device__ constexpr int gather_rows(int d) { return GATHER_THREADS / (d / 8) * GATHER_PASSES; }

template <int D, bool BY_VALUE>
__global__ void __launch_bounds__(GATHER_THREADS) attn_gather_rows_kernel(EvictArgs a, PlanWords<BY_VALUE> words) {
    constexpr int CPR = D / 8, STEP = GATHER_THREADS / CPR;
    const EvictPlan e(BY_VALUE ? words.w : a.plan, a.n_req);
    const int kvh = (int)blockIdx.x % a.H_kv, block = (int)blockIdx.x / a.H_kv;
    const int r = __builtin_amdgcn_readfirstlane(request_of(e.block_cu, a.n_req, block));
    const int keep = e.keep[r], mask = (1 << a.page_shift) - 1;
    const int32_t* const index = a.index + (int64_t)a.H_kv * e.keep_cu[r] + (int64_t)kvh * keep;
    const int32_t *const ids = e.page_ids + e.place[r], *const new_ids = e.page_ids + e.new_place[r];
    const int to0 = (block - e.block_cu[r]) * gather_rows(D) + (int)threadIdx.x / CPR, c = (int)threadIdx.x % CPR;
    const int64_t head = (int64_t)kvh << a.page_shift;
    int from[GATHER_PASSES];
    int64_t old_page[GATHER_PASSES], new_page[GATHER_PASSES];
#pragma unroll
    for (int i = 0; i < GATHER_PASSES; ++i) {
        const int to = min(to0 + i * STEP, keep - 1);
        from[i] = index[to];
        new_page[i] = new_ids[to >> a.page_shift];
    }
#pragma unroll
    for (int i = 0; i < GATHER_PASSES; ++i) old_page[i] = ids[from[i] >> a.page_shift];
    u32x4 k[GATHER_PASSES], v[GATHER_PASSES];
    float w[GATHER_PASSES];
#pragma unroll
    for (int i = 0; i < GATHER_PASSES; ++i) {
        const int64_t src = old_page[i] * a.page_stride + (head + (from[i] & mask)) * D + 8 * c;
        k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.k_pool + src));
        v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.v_pool + src));
        if (c == 0) w[i] = a.w_pool[old_page[i] * a.w_stride + head + (from[i] & mask)];
    }
#pragma unroll
    for (int i = 0; i < GATHER_PASSES; ++i) {
        const int to = to0 + i * STEP;
        if (to >= keep) break;
        const int64_t dst = new_page[i] * a.page_stride + (head + (to & mask)) * D + 8 * c;
        __builtin_nontemporal_store(k[i], reinterpret_cast<u32x4*>(a.k_pool + dst));
        __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(a.v_pool + dst));
        if (c == 0) a.w_pool[new_page[i] * a.w_stride + head + (to & mask)] = w[i];
    }
}

}  // namespace attn
