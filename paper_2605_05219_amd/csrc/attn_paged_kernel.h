// Device side of the paged cache's own operators (see include/attn_paged.h): rotary positions with the append, the attention weight
// that cached rows gather, and eviction by it.  The attention over the pages is attn_kernel.h's, with PagedArgs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_kernel.h"

namespace attn {

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

struct RopeArgs {
    const void *q, *k, *v;
    uint16_t* q_out;
    uint16_t *k_pool, *v_pool;
    const int32_t *cu, *start, *pos, *place, *page_ids;   // place: where the page of row 0 would be listed
    int64_t ldq, ldk, ldv, page_stride;
    int32_t n_req, T, tokens;         // tokens: per workgroup
    int32_t H_q, H_kv, units;         // units: pieces of 16 elements per head, d / 16
    int32_t page_shift, rot, layout;
    float amplitude;
    uint64_t turn[128];               // turns per position, 2^-64
};

template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, float* x) {
    if constexpr (F32) {
        const f32x4* const s = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
        const f32x4 a = s[0], b = s[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, a[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
        }
    }
}
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

// One workgroup takes `tokens` tokens: their cosines and sines once, to LDS, for all heads; then one thread per 16 elements of a
// head (two runs of 8 where a pair's halves lie apart).
template <bool F32>
__global__ void __launch_bounds__(ROPE_THREADS) attn_rope_kernel(RopeArgs a) {
    __shared__ float cs[ROPE_TOKENS][2][128];
    __shared__ int64_t row_at[ROPE_TOKENS];      // the token's row in the pools, head 0
    __shared__ int32_t position[ROPE_TOKENS];
    const int tok0 = (int)blockIdx.x * a.tokens;
    const int n_tok = min(a.tokens, a.T - tok0);
    const int wave = threadIdx.x >> 6;
    const int D = 16 * a.units;
    for (int i = wave; i < n_tok; i += ROPE_THREADS / 64) {
        const int t = tok0 + i, r = request_of(a.cu, a.n_req, t);
        if ((threadIdx.x & 63) == 0) {
            const int in = t - a.cu[r], row = a.start[r] + in;
            position[i] = a.pos[r] + in;
            row_at[i] = (int64_t)a.page_ids[a.place[r] + (row >> a.page_shift)] * a.page_stride + (int64_t)(row & ((1 << a.page_shift) - 1)) * D;
        }
    }
    __syncthreads();
    const int half = a.rot >> 1;
    for (int i = threadIdx.x; i < n_tok * half; i += ROPE_THREADS) {
        const int t = i / half, p = i - t * half;
        const uint64_t turns = (uint64_t)(uint32_t)position[t] * a.turn[p];
        float sn, cn;
        sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &sn, &cn);
        cs[t][0][p] = cn * a.amplitude;
        cs[t][1][p] = sn * a.amplitude;
    }
    __syncthreads();
    const int heads = a.H_q + 2 * a.H_kv, per = heads * a.units;
    for (int i = threadIdx.x; i < n_tok * per; i += ROPE_THREADS) {
        const int t = i / per, j = i - t * per;
        const int head = j / a.units, u = j - head * a.units;
        const int64_t tok = tok0 + t;
        float x[16];
        if (head >= a.H_q + a.H_kv) {            // a value: widened
            const int h = head - a.H_q - a.H_kv;
            const int64_t src = tok * a.ldv + h * D + 16 * u;
            load8<F32>(a.v, src, x);
            load8<F32>(a.v, src + 8, x + 8);
            uint16_t* const dst = a.v_pool + row_at[t] + ((int64_t)h * D << a.page_shift) + 16 * u;
            store8_fp16(dst, x);
            store8_fp16(dst + 8, x + 8);
            continue;
        }
        const bool key = head >= a.H_q;
        const int h = key ? head - a.H_q : head;
        const bool turned = 16 * u < a.rot, apart = turned && a.layout == 0;
        const int lo = apart ? 8 * u : 16 * u, hi = apart ? half + 8 * u : 16 * u + 8;
        const int64_t src = (key ? tok * a.ldk : tok * a.ldq) + h * D;
        const void* const from = key ? a.k : a.q;
        load8<F32>(from, src + lo, x);
        load8<F32>(from, src + hi, x + 8);
        if (turned) {
            float y[16];
            if (apart) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float cn = cs[t][0][8 * u + e], sn = cs[t][1][8 * u + e];
                    y[e] = x[e] * cn - x[8 + e] * sn;
                    y[8 + e] = x[8 + e] * cn + x[e] * sn;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float cn = cs[t][0][8 * u + e], sn = cs[t][1][8 * u + e];
                    y[2 * e] = x[2 * e] * cn - x[2 * e + 1] * sn;
                    y[2 * e + 1] = x[2 * e + 1] * cn + x[2 * e] * sn;
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = y[e];
        }
        uint16_t* const dst = key ? a.k_pool + row_at[t] + ((int64_t)h * D << a.page_shift) : a.q_out + (tok * a.H_q + h) * D;
        store8_bf16(dst + lo, x);
        store8_bf16(dst + hi, x + 8);
    }
}

// ---------------------------------------------------------------- the weight that cached rows gather
// A key's sum runs over query rows, so keys stay and queries pass: each of the four waves of a workgroup holds 64 keys in registers as
// matrix operands, tiles of 32 query rows (tokens x heads of the group, row = token * G + head) go through two LDS stages, brought by loads to LDS a
// tile ahead.  S[row][key] puts a key into a lane's column and 16 of the rows into its registers: the sum over rows needs no
// exchange between lanes but one with the other half at the end, and no atomics.  A row's log-sum-exp comes by LDS in units of log2.
constexpr int WGT_THREADS = 256;
constexpr int WGT_KEYS = 256;         // keys per workgroup
constexpr int WGT_ROWS = 32;          // query rows per tile
constexpr int WGT_PARTS = 2048;       // (tile, part, head) triples of calls that cut the rows of a tile into parts, at most

struct WeightArgs {
    const uint16_t* q;
    const float* lse;
    const uint16_t* k_pool;
    const float* w_in;        // or nullptr
    float* w_out;
    const int32_t *cu, *start, *place, *page_ids;
    const int32_t* block_cu;  // n_req + 1: (key tile, part) pairs before each request
    float* part;              // [pair][head][WGT_KEYS], where a request's rows are cut
    int64_t page_stride, w_stride;
    int32_t n_req, H_q, H_kv, G;
    int32_t page_shift;
    int32_t part_rows;        // query rows per part, a multiple of WGT_ROWS
    float scale_log2e, decay;
};

template <int D>
struct WeightSmem {
    static constexpr int CPR = D / 8, ROW_BYTES = D * 2, TILE_BYTES = WGT_ROWS * ROW_BYTES;
    static constexpr int PPW = TILE_BYTES / 4096;       // 1 KiB loads per wave and tile
    static __device__ __forceinline__ int f(int row) { return CPR >= 16 ? (row & 15) : ((row >> 1) & 7); }
};

__device__ __forceinline__ void store_weight(const WeightArgs& a, int place, int kvh, int c0, int key, float sum) {
    const int64_t at = (int64_t)a.page_ids[place + (key >> a.page_shift)] * a.w_stride + ((int64_t)kvh << a.page_shift) + (key & ((1 << a.page_shift) - 1));
    a.w_out[at] = (a.w_in && key < c0 ? a.decay * a.w_in[at] : 0.f) + sum;
}

template <int D>
__global__ void __launch_bounds__(WGT_THREADS) attn_weights_kernel(WeightArgs a) {
    typedef WeightSmem<D> SM;
    constexpr int KB = D / 16;
    __shared__ __attribute__((aligned(1024))) char stage0[SM::TILE_BYTES], stage1[SM::TILE_BYTES];
    __shared__ __attribute__((aligned(16))) float neg_lse[2][WGT_ROWS];   // -lse log2(e); rows past the end -inf
    __shared__ __attribute__((aligned(16))) int limit[2][WGT_ROWS];       // last key a row sees

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, g = lane >> 5;
    const int kvh = (int)blockIdx.x % a.H_kv, pair = (int)blockIdx.x / a.H_kv;
    const int r = request_of(a.block_cu, a.n_req, pair);
    const int tok0 = a.cu[r], n = a.cu[r + 1] - tok0, c0 = a.start[r], place = a.place[r];
    const int kv_len = c0 + n, rows = n * a.G;
    const int parts = max(1, (rows + a.part_rows - 1) / a.part_rows);
    const int in_req = pair - a.block_cu[r];
    const int kv0 = in_req / parts * WGT_KEYS, part = in_req % parts;
    const int seen_from = max(0, kv0 - c0) * a.G / WGT_ROWS * WGT_ROWS;   // the first rows that see a key of this tile
    const int row_lo = max(part * a.part_rows, seen_from), row_hi = min((part + 1) * a.part_rows, rows);

    // ---- this wave's keys: operand B, column = key, d = 16 kb + 8 g + {0..7}
    const int key0 = kv0 + 64 * wave;
    bf16x8 kf[2][KB];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int key = min(key0 + 32 * b + col, kv_len - 1);
        const uint16_t* const kp = a.k_pool + (int64_t)a.page_ids[place + (key >> a.page_shift)] * a.page_stride + ((int64_t)kvh * D << a.page_shift) +
                                   (int64_t)(key & ((1 << a.page_shift) - 1)) * D + 8 * g;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) kf[b][kb] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(kp + 16 * kb));
    }

    // ---- a tile of query rows from `row`: to LDS, 16-byte chunk c of a row at c ^ f(row)
    auto issue = [&](int row, char* sb) {
        const int t_lo = min(row, rows - 1) / a.G, t_hi = min(row + WGT_ROWS - 1, rows - 1) / a.G;
        const uint16_t* const base = a.q + ((int64_t)(tok0 + t_lo) * a.H_q + kvh * a.G) * D;
        const int bytes = ((t_hi - t_lo) * a.H_q + a.G) * D * 2;
#pragma unroll
        for (int i = 0; i < SM::PPW; ++i) {
            const int s = (wave * SM::PPW + i) * 64 + lane, rr = s / SM::CPR, pos = s % SM::CPR;
            const int rho = min(row + rr, rows - 1), t = rho / a.G;
            load_to_lds(base, bytes, sb + (wave * SM::PPW + i) * 1024, ((t - t_lo) * a.H_q + rho - t * a.G) * D * 2 + ((pos ^ SM::f(rr)) << 4), 0);
        }
    };
    auto stage_rows = [&](int row, int st) {             // by 32 threads
        const int rho = min(row + (int)threadIdx.x, rows - 1), t = rho / a.G;
        const float x = a.lse[(int64_t)(tok0 + t) * a.H_q + kvh * a.G + rho - t * a.G];
        neg_lse[st][threadIdx.x] = row + (int)threadIdx.x < row_hi ? -x * 1.4426950408889634f : -INFINITY;
        limit[st][threadIdx.x] = c0 + t;
    };
    float acc[2] = {0.f, 0.f};
    auto tile = [&](int row, int st, const char* sb, char* other) {
        wait_vmcnt<0>();
        __syncthreads();
        if (row + WGT_ROWS < row_hi) issue(row + WGT_ROWS, other);
        f32x16 S[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[b][i] = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const bf16x8 qf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(sb + col * SM::ROW_BYTES + (((2 * kb + g) ^ SM::f(col)) << 4)));
#pragma unroll
            for (int b = 0; b < 2; ++b) S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[b][kb], S[b], 0, 0, 0);
        }
        const bool cut = c0 + row / a.G < key0 + 63;      // some row does not see some key of this wave
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 nl = *reinterpret_cast<const f32x4*>(&neg_lse[st][8 * q + 4 * g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int lim = cut ? limit[st][8 * q + 4 * g + e] : INT32_MAX;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(S[b][4 * q + e], a.scale_log2e, nl[e]));
                    acc[b] += key0 + 32 * b + col <= lim ? p : 0.f;
                }
            }
        }
        if (row + WGT_ROWS < row_hi && threadIdx.x < WGT_ROWS) stage_rows(row + WGT_ROWS, st ^ 1);
    };
    if (row_lo < row_hi) {
        issue(row_lo, stage0);
        if (threadIdx.x < WGT_ROWS) stage_rows(row_lo, 0);
        for (int row = row_lo; row < row_hi; row += 2 * WGT_ROWS) {
            tile(row, 0, stage0, stage1);
            if (row + WGT_ROWS < row_hi) tile(row + WGT_ROWS, 1, stage1, stage0);
        }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const float sum = sum_with_other_half(acc[b]);
        const int key = key0 + 32 * b + col;
        if (g != 0 || key >= kv_len) continue;
        if (parts == 1) store_weight(a, place, kvh, c0, key, sum);
        else a.part[((int64_t)pair * a.H_kv + kvh) * WGT_KEYS + key - kv0] = sum;
    }
}

// The parts of a tile's rows, summed in order; one workgroup per (tile, head) and one thread per key.  tile_cu: tiles of cut requests
// before each request.
__global__ void __launch_bounds__(WGT_KEYS) attn_weights_merge_kernel(WeightArgs a, const int32_t* tile_cu) {
    const int kvh = (int)blockIdx.x % a.H_kv, tile = (int)blockIdx.x / a.H_kv;
    const int r = request_of(tile_cu, a.n_req, tile);
    const int tok0 = a.cu[r], n = a.cu[r + 1] - tok0, c0 = a.start[r];
    const int parts = (n * a.G + a.part_rows - 1) / a.part_rows;
    const int in_req = tile - tile_cu[r], key = in_req * WGT_KEYS + (int)threadIdx.x;
    if (key >= c0 + n) return;
    float sum = 0.f;
    for (int p = 0; p < parts; ++p) sum += a.part[(((int64_t)a.block_cu[r] + (int64_t)in_req * parts + p) * a.H_kv + kvh) * WGT_KEYS + threadIdx.x];
    store_weight(a, a.place[r], kvh, c0, key, sum);
}

// ---------------------------------------------------------------- eviction
struct EvictArgs {
    uint16_t *k_pool, *v_pool;
    float* w_pool;
    int32_t* index;
    const int32_t *rows, *keep, *first, *recent;          // keep: at most rows
    const int32_t *place, *new_place, *keep_cu, *page_ids;   // page_ids: old and new ones; keep_cu: kept rows before each request
    int64_t page_stride, w_stride;
    int32_t n_req, H_kv, page_shift;
    int32_t chunks;                                       // 16-byte chunks per row, d / 8
};
constexpr int SEL_THREADS = 1024;
constexpr int GATHER_THREADS = 256;

// A weight's rank as an unsigned number: larger weights larger, -0 as +0, what is not a number 0.
__device__ __forceinline__ uint32_t weight_rank(float w) {
    if (w != w) return 0u;
    const uint32_t u = __builtin_bit_cast(uint32_t, w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The rows that one (request, head) keeps.  Four rounds over 8 bits each of the rank find the smallest rank kept and how many rows of
// just that rank are; a last pass over the rows in order writes the row numbers kept.
__global__ void __launch_bounds__(SEL_THREADS) attn_select_kernel(EvictArgs a) {
    constexpr int WAVES = SEL_THREADS / 64;
    __shared__ int hist[256];
    __shared__ uint32_t found[2];        // prefix of the smallest rank kept, rows of it still to take
    __shared__ int wave_sum[2][WAVES];
    const int r = (int)blockIdx.x / a.H_kv, kvh = (int)blockIdx.x % a.H_kv;
    const int rows = a.rows[r], keep = a.keep[r], first = a.first[r], last = rows - a.recent[r];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t* const ids = a.page_ids + a.place[r];
    auto rank_of = [&](int j) {
        return weight_rank(a.w_pool[(int64_t)ids[j >> a.page_shift] * a.w_stride + ((int64_t)kvh << a.page_shift) + (j & ((1 << a.page_shift) - 1))]);
    };
    const int want = keep - first - a.recent[r];          // rows to take from [first, last)
    uint32_t prefix = 0;
    int left = want;
    if (keep < rows && want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int j = first + tid; j < last; j += SEL_THREADS) {
                const uint32_t x = rank_of(j);
                if (shift == 24 || x >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[(x >> shift) & 255], 1);
            }
            __syncthreads();
            if (wave == 0) {                              // from the largest digit down: lane l has digits 255 - 4 l .. 252 - 4 l
                int c[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - 4 * lane - i];
                int before = sum;
                for (int d = 1; d < 64; d <<= 1) {
                    const int up = __shfl_up(before, d);
                    if (lane >= d) before += up;
                }
                before -= sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < left && before + c[i] >= left) {
                        found[0] = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
                        found[1] = (uint32_t)(left - before);
                    }
                    before += c[i];
                }
            }
            __syncthreads();
            prefix = found[0];
            left = (int)found[1];
            __syncthreads();
        }
    }
    // ---- the rows kept, in order
    int32_t* const out = a.index + (int64_t)a.H_kv * a.keep_cu[r] + (int64_t)kvh * keep;
    int kept = 0, ties = 0;
    for (int j0 = 0; j0 < rows; j0 += SEL_THREADS) {
        const int j = j0 + tid;
        const bool always = j < rows && (keep == rows || j < first || j >= last);
        const bool middle = j < rows && !always && want > 0;
        const uint32_t x = middle ? rank_of(j) : 0u;
        const bool tie = middle && x == prefix;
        const uint64_t tie_mask = __ballot(tie);
        const uint64_t below = (1ull << lane) - 1;
        if (lane == 0) wave_sum[0][wave] = __popcll(tie_mask);
        __syncthreads();
        int tie_at = ties, tie_all = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) tie_at += wave_sum[0][w];
            tie_all += wave_sum[0][w];
        }
        tie_at += __popcll(tie_mask & below);
        const bool take = always || (middle && (x > prefix || (tie && tie_at < left)));
        const uint64_t mask = __ballot(take);
        if (lane == 0) wave_sum[1][wave] = __popcll(mask);
        __syncthreads();
        int at = kept, all = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) at += wave_sum[1][w];
            all += wave_sum[1][w];
        }
        if (take) out[at + __popcll(mask & below)] = j;
        kept += all;
        ties += tie_all;
        __syncthreads();
    }
}

// The kept rows go to the new pages: one thread per 16-byte chunk of k and of v, a row's first one its weight too.
__global__ void __launch_bounds__(GATHER_THREADS) attn_gather_rows_kernel(EvictArgs a, int64_t n) {
    const int64_t id = (int64_t)blockIdx.x * GATHER_THREADS + threadIdx.x;
    if (id >= n) return;
    const int64_t item = id / a.chunks;                   // index entry
    const int c = (int)(id - item * a.chunks);
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)a.keep_cu[mid] * a.H_kv <= item) lo = mid; else hi = mid;
    }
    const int r = lo, keep = a.keep[r];
    const int64_t in = item - (int64_t)a.keep_cu[r] * a.H_kv;
    const int kvh = (int)(in / keep), to = (int)(in - (int64_t)kvh * keep), from = a.index[item];
    const int mask = (1 << a.page_shift) - 1;
    const int64_t p0 = a.page_ids[a.place[r] + (from >> a.page_shift)], p1 = a.page_ids[a.new_place[r] + (to >> a.page_shift)];
    const int64_t head = (int64_t)kvh << a.page_shift;
    const int64_t src = p0 * a.page_stride + ((head + (from & mask)) * a.chunks + c) * 8;
    const int64_t dst = p1 * a.page_stride + ((head + (to & mask)) * a.chunks + c) * 8;
    *reinterpret_cast<u32x4*>(a.k_pool + dst) = *reinterpret_cast<const u32x4*>(a.k_pool + src);
    *reinterpret_cast<u32x4*>(a.v_pool + dst) = *reinterpret_cast<const u32x4*>(a.v_pool + src);
    if (c == 0) a.w_pool[p1 * a.w_stride + head + (to & mask)] = a.w_pool[p0 * a.w_stride + head + (from & mask)];
}

}  // namespace attn
