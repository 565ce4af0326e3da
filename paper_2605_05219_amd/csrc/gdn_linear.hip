// gdn_linear: the layers' projections y = x w^T + bias on the bf16 matrix cores (see include/gdn_linear.h).
//
// One workgroup of four or eight waves makes a BM (tokens) x BN (outputs) tile, a wave its part of it as tiles of
// v_mfma_f32_16x16x32_bf16.  Both operands are read along k, so a k step of BK needs a BM x BK tile of x and a
// BN x BK tile of w; they come from memory with 16-byte buffer loads straight to LDS (no registers) into a ring of
// STAGES stages, STAGES - 1 k steps ahead of the matrix cores: one barrier per k step.  The shapes that are built:
//   0: 128 x 128 x 64, 2 stages, four waves, two workgroups per compute unit   many small tiles: one workgroup's waits under the other's products
//   1: 256 x 256 x 64, 2 stages, four waves, one workgroup per compute unit: a wave holds 128 x 128 outputs in 256
//      accumulator registers: fewer operand bytes from LDS per flop, one wave per SIMD (kept for comparison: within 3 % of 2 either way)
//   2: 256 x 256 x 64, 2 stages, eight waves of 128 tokens x 64 outputs, two per SIMD: while one wave of a SIMD is held up
//      issuing its loads to LDS the other feeds the matrix pipe, and a barrier covers 64 of k (the default for large problems)
//   3: 64 x 64 x 64, 5 stages, four waves of 32 x 32 outputs, two workgroups per compute unit: problems whose 64 x 64 tiles fit
//      the chip in one round, where a larger tile would walk k on too few compute units (512 x 2048 x 2048 9.9 us against 16 of
//      shape 4 and 21 of shape 0)
//   4: 128 x 128 x 64, 4 stages, eight waves, one workgroup per compute unit: problems of at most one round of such tiles are bound by
//      the latency of a k step's loads (0.9 us where the weights come from memory), of which this shape has three in flight
//      (384 x 8224 x 2048 23 us against 31 of shape 0)
//   5: 128 x 160 x 64, 4 stages, four waves, one workgroup per compute unit: the same for problems that shape 4 just does not
//      fit in one round (512 x 8224: 260 tiles of 128 outputs for 256 compute units, 208 of 160; 27 us against 36 of shape 4, 32 of shape 0)
// The same tiles make gdn_linear_act's products, with the activation, gate, factor and residual between the sums and the store (act_epilogue), and those of a mixture
// of experts, on rows that a list names (launch_expert_product).  For at most 1024 rows gdn_linear_act has six kernels more, shapes 6 to 11 (gdn_few_kernel.h).
//   8192 x 2 x 6144 x 2048 with SiLU and gate 304 to 325 us by card (1270 to 1355 TFLOP/s; a library product of 8192 x 12288 x 2048 alone 361), the activation under 3 % of it;
//   8192 x 2048 x 6144 onto the stream, the way back, 168 us with it in bf16, 180 in fp32 (1226, 1147 TFLOP/s; a library product alone 141), 2048 rows onto fp32 53 (52);
//   1401 x 1733 x 1600 with GELU, an fp32 residual and fp32 outputs 21.6: 10 of them its 25 k steps (what a compute unit is sent, 80 GB/s), 2.5 the GELU, 1.6 the residual,
//   8 the beginning and the end of one round of 154 tiles (shape 0 35, 3 25.7, 5 36; three workgroups of shape 3 with three stages each 23.8, tiles of 96 x 128 24.7).
// The products are v_mfma_f32_16x16x32_bf16: half the accumulator traffic per flop of the 32 x 32 x 16 instruction, at the same rate on
// paper; on a chip held by its power limit 8192 x 2048 x 2048 takes 51 us with it and 56 with the other, 512 x 2048 10.4 and 12.3.
// A load to LDS writes a wave's 1 KiB contiguously (lane i at 16 i), so rows are unpadded (2 BK bytes) and bank
// conflicts are avoided by choosing WHICH 16-byte piece of its row a lane fetches: piece p of row r is stored at
// position p ^ swz(r), swz(r) = (r / rows per 256 bytes) % pieces per row, which makes the 16 lanes that read the
// same piece of 16 consecutive rows hit 16 different 16-byte bank groups.  Rows past the end of x or w read as
// zeros (the buffer descriptor ends with the matrix); they only feed outputs that are never stored.  The products
// are taken transposed (w rows as the left operand), so that a lane holds four consecutive outputs of ONE token
// and writes them to LDS, for the turn to whole rows, with one 8- or 16-byte store.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "gdn_act.h"
#include "gdn_few_kernel.h"
#include "gdn_linear.h"
#include "gdn_linear_tiles.h"
#include "gdn_rows.h"

namespace gdn {
namespace linear {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));


constexpr int LIN_MAX_SEG = 8;

struct LinearArgs {
    const void* x;
    const void* w;
    const float* bias;
    void* y;
    int64_t ldx, ldw, ldy;
    int64_t T;
    int32_t N, K;
    int32_t tiles_m, tiles_n;
    int32_t per_xcd;                    // tiles per XCD
    // gdn_linear_split: the outputs go to n_seg destinations by column range; n_seg = 0: everything to y
    int32_t n_seg;
    int32_t seg_col[LIN_MAX_SEG + 1];   // segment s holds outputs seg_col[s] .. seg_col[s + 1] - 1
    void* seg_y[LIN_MAX_SEG];
    int64_t seg_ld[LIN_MAX_SEG];
};

// gdn_linear_act: what its epilogue does beside the bias
struct LinearActArgs : LinearArgs {
    const void* w_up;                   // null: one product
    const float* bias_up;
    const void* residual;
    int64_t ldw_up, ldr;
    int32_t act, res_f32;
    float scale;
};
// What a kernel makes of its sums: the bias added; with an activation, a factor and a residual; the same of two products, in the tiles of
// 16 outputs in turn (a wave's output tile 2 p holds 16 outputs of the gate, 2 p + 1 the same of w_up: one lane has both).
// The experts' products are the second and the third of these on rows that a list names (gdn_linear_tiles.h).
enum { EPI_BIAS = 0, EPI_ACT = 1, EPI_GATED = 2, EPI_EXPERT = 3, EPI_EXPERT_GATED = 4 };
constexpr bool epi_gated(int e) { return e == EPI_GATED || e == EPI_EXPERT_GATED; }
constexpr bool epi_expert(int e) { return e >= EPI_EXPERT; }
struct ExpertArgs : LinearActArgs {
    const int32_t* list;
    const ExpertTile* table;
    const int32_t* n_tiles;
    const float* weights;
    int32_t list_stride, div, x_rows;
};
template <int EPI> struct EpiArgs { typedef ExpertArgs type; };
template <> struct EpiArgs<EPI_BIAS> { typedef LinearArgs type; };
template <> struct EpiArgs<EPI_ACT> { typedef LinearActArgs type; };
template <> struct EpiArgs<EPI_GATED> { typedef LinearActArgs type; };

inline int32_t hip_err(hipError_t e) { return e == hipSuccess ? GDN_OK : GDN_ERR_HIP - (int32_t)e; }

// s_waitcnt vmcnt(N) (gfx9 encoding: vmcnt in bits 3:0 and 15:14; other counters left alone)
template <int N>
__device__ __forceinline__ void wait_vm() {
    __builtin_amdgcn_s_waitcnt(((N & 0x30) << 10) | (N & 0xF) | 0x0F70);
}

template <int BM_, int BN_, int BK_, int STAGES_, int WGS_PER_CU_, int WAVES_M_, int WAVES_N_>
struct LinCfg {
    static constexpr int BM = BM_, BN = BN_, BK = BK_, STAGES = STAGES_, WGS_PER_CU = WGS_PER_CU_;
    static constexpr int WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, NW = WAVES_M * WAVES_N, THREADS = 64 * NW;   // the wave grid over the tile
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N;   // a wave's tokens and outputs
    static constexpr int RB = BK * 2;                  // bytes of a tile row
    static constexpr int PP = RB / 16;                 // 16-byte pieces per row
    static constexpr int RL = 256 / RB;                // rows per 256 bytes (the span of the 64 banks)
    static constexpr int ROWS_PER_LOAD = 1024 / RB;    // rows a wave-wide load covers
    static constexpr int X_BYTES = BM * RB, W_BYTES = BN * RB, STAGE_BYTES = X_BYTES + W_BYTES;
    static constexpr int SMEM = STAGES * STAGE_BYTES;
    static constexpr int TI = WM / 16, TJ = WN / 16;   // 16 x 16 tiles of a wave along tokens / outputs
    static constexpr int XL = BM / ROWS_PER_LOAD / NW, WL = BN / ROWS_PER_LOAD / NW;   // loads per wave and stage
    static constexpr int LPS = XL + WL;
    static constexpr int AHEAD = (STAGES - 2) * LPS;   // loads that may still be in flight when a stage is handed over
    static_assert(PP * RL == 16 && (STAGES - 1) * LPS < 64 && SMEM * WGS_PER_CU <= 160 * 1024 && (BK / 32) % 2 == 0 &&
                  XL * ROWS_PER_LOAD * NW == BM && WL * ROWS_PER_LOAD * NW == BN && TI * 16 == WM && TJ * 16 == WN, "tile shape");
};
typedef LinCfg<128, 128, 64, 2, 2, 2, 2> LinSmall;
typedef LinCfg<256, 256, 64, 2, 1, 2, 2> LinBig;      // four waves, 128 x 128 outputs each
typedef LinCfg<256, 256, 64, 2, 1, 2, 4> LinBig8;     // eight waves, 128 tokens x 64 outputs each: two waves per SIMD
typedef LinCfg<64, 64, 64, 5, 2, 2, 2> LinTiny;       // four waves of 32 x 32 outputs each, four k steps of 64 in flight
typedef LinCfg<64, 64, 64, 3, 3, 2, 2> LinTiny3;      // the experts' where k is short: a third workgroup's products under the others' first loads and outputs
typedef LinCfg<128, 128, 64, 4, 1, 2, 4> LinDeep;     // eight waves, 64 x 32 outputs each, three k steps of 64 in flight
typedef LinCfg<128, 160, 64, 4, 1, 2, 2> LinWide;     // four waves, 64 x 80 outputs each, three k steps of 64 in flight

// The loads of one wave for one stage: 1 KiB each, XL of its quarter of the x tile, then WL of the w tile.
template <typename CFG>
struct LinLoad {
    static __device__ __forceinline__ void one(int j, char* smem, int stage, int k0, int wave, const char* xb, int x_bytes, const char* wb,
                                               int w_bytes, const int* xoff, const int* woff) {
        // buffer descriptors that end with the matrices: rows past T or N arrive as zeros
        char* xs = smem + stage * CFG::STAGE_BYTES;
        char* ws = xs + CFG::X_BYTES;
        if (j < CFG::XL) {
            const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(xb), 0, x_bytes, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)(xs + ((CFG::BM / CFG::NW) * wave + CFG::ROWS_PER_LOAD * j) * CFG::RB), 16, xoff[j], k0 * 2, 0, 0);
        } else {
            const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(wb), 0, w_bytes, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (__attribute__((address_space(3))) void*)(ws + ((CFG::BN / CFG::NW) * wave + CFG::ROWS_PER_LOAD * (j - CFG::XL)) * CFG::RB), 16, woff[j - CFG::XL], k0 * 2, 0, 0);
        }
    }
};

// Which of the two weights the wave's load j belongs to, where tiles of 16 rows take turns (a load's rows lie in one of them).
template <typename CFG>
__device__ __forceinline__ bool up_load(int j, int wave) {
    return (((CFG::BN / CFG::NW) * wave + CFG::ROWS_PER_LOAD * j) >> 4) & 1;
}

// One bias, activation, factor and residual on a wave's outputs, and out through LDS in fp32 (one rounding, behind the residual): as
// the epilogue below, a row of at most 64 outputs to a pass.
template <typename CFG, bool OUT_BF16, int EPI>
__device__ __forceinline__ void act_epilogue(const typename EpiArgs<EPI>::type& a, f32x4 (&acc)[CFG::TJ][CFG::TI], char* reg, int64_t tok0, int col0,
                                             int lane, const int32_t* list, int64_t n_rows) {
    constexpr int PAIR = epi_gated(EPI) ? 2 : 1;                 // accumulator tiles to a tile of outputs
    constexpr int WN = CFG::WN / PAIR, WM = CFG::WM;
    constexpr int REGION = CFG::SMEM / CFG::NW;
    constexpr int PW = WN <= 64 ? WN : 16;                         // outputs per pass (shape 5's 80 go 16 at a time)
    constexpr int RBY = PW * 4 <= 64 ? 64 : PW * 4 <= 128 ? 128 : 256, PPR = RBY / 16;
    constexpr int TP = WM * RBY <= REGION ? WM : REGION / RBY >= 64 ? 64 : REGION / RBY >= 32 ? 32 : 16;
    constexpr int OPL = OUT_BF16 ? 8 : 4;                          // outputs of a lane's store
    constexpr int LPR = PW / OPL, RPI = 64 / LPR, IT = TP / RPI;  // lanes per row, rows a wave-wide store covers, stores of a pass
    static_assert(TP * RBY <= REGION && TP % RPI == 0 && WM % TP == 0 && WN % PW == 0 && PW % 16 == 0 && CFG::TJ % PAIR == 0, "epilogue region");
    const int lr = lane & 15, g = lane >> 4;
#pragma unroll
    for (int c0 = 0; c0 < WN; c0 += PW) {
#pragma unroll
        for (int t0 = 0; t0 < WM; t0 += TP) {
            // the pass's residual goes out in front of the activations, whose time covers its latency
            u32x4 res[IT][2];
            if (!epi_expert(EPI) && a.residual) {
#pragma unroll
                for (int i = 0; i < IT; ++i) {
                    const int64_t tok = tok0 + t0 + RPI * i + lane / LPR;
                    const int col = col0 + c0 + lane % LPR * OPL;
                    if (tok >= n_rows || col + OPL > a.N) continue;      // (the last columns below)
                    if (a.res_f32) {
                        const u32x4* r = reinterpret_cast<const u32x4*>(static_cast<const float*>(a.residual) + tok * a.ldr + col);
                        res[i][0] = r[0];
                        if (OUT_BF16) res[i][1] = r[1];
                    } else if (OUT_BF16) {
                        res[i][0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.residual) + tok * a.ldr + col);
                    } else {
                        const uint2 r = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.residual) + tok * a.ldr + col);
                        res[i][0][0] = r.x;
                        res[i][0][1] = r.y;
                    }
                }
            }
#pragma unroll
            for (int tj = c0 / 16; tj < (c0 + PW) / 16; ++tj) {
                const int cl = 16 * tj + 4 * g;
                f32x4 bv = {0.f, 0.f, 0.f, 0.f}, bu = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col0 + cl + e < a.N) {
                        if (a.bias) bv[e] = a.bias[col0 + cl + e];
                        if (epi_gated(EPI) && a.bias_up) bu[e] = a.bias_up[col0 + cl + e];
                    }
#pragma unroll
                for (int ti = t0 / 16; ti < (t0 + TP) / 16; ++ti) {
                    const int row = 16 * ti + lr - t0;
                    f32x4 v = activate(a.act, acc[PAIR * tj][ti] + bv);
                    if (epi_gated(EPI)) v *= acc[PAIR * tj + PAIR - 1][ti] + bu;
                    const int piece = (cl - c0) / 4;
                    *reinterpret_cast<f32x4*>(reg + row * RBY + ((piece ^ (row % PPR)) << 4)) = v;
                }
            }
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int row = RPI * i + lane / LPR, first = lane % LPR * OPL;
                f32x4 v[OPL / 4];
#pragma unroll
                for (int h = 0; h < OPL / 4; ++h)
                    v[h] = *reinterpret_cast<const f32x4*>(reg + row * RBY + (((first / 4 + h) ^ (row % PPR)) << 4));
                int64_t tok = tok0 + t0 + row;
                const int col = col0 + c0 + first;
                if (tok >= n_rows || col + OPL > a.N) continue;
                float scale = a.scale;
                if constexpr (epi_expert(EPI)) {
                    // (an expert's inner row, weighted, is rounded to bf16 below: the second product's operand on the bf16 matrix cores.  Whole, it would be two operands, twice that
                    // product's instructions and twice the bytes here; so y is off by 2.3e-3 (norms, against 64 bits), of which its own rounding is 1.7e-3)
                    tok = list[tok];
                    if (EPI == EPI_EXPERT_GATED) scale = a.weights[tok];
                }
#pragma unroll
                for (int h = 0; h < OPL / 4; ++h) v[h] *= scale;
                if (!epi_expert(EPI) && a.residual) {
                    if (a.res_f32) {
#pragma unroll
                        for (int h = 0; h < OPL / 4; ++h) v[h] += __builtin_bit_cast(f32x4, res[i][h]);
                    } else {
#pragma unroll
                        for (int e = 0; e < OPL; ++e)
                            v[e / 4][e % 4] += __uint_as_float(e & 1 ? res[i][0][e / 2] & 0xffff0000u : res[i][0][e / 2] << 16);
                    }
                }
                char* const p = static_cast<char*>(a.y) + (tok * a.ldy + col) * (OUT_BF16 ? 2 : 4);
                if (OUT_BF16) {
                    bf16x8 o;
#pragma unroll
                    for (int e = 0; e < OPL; ++e) o[e] = (__bf16)v[e / 4][e % 4];
                    *reinterpret_cast<bf16x8*>(p) = o;
                } else {
                    *reinterpret_cast<f32x4*>(p) = v[0];
                }
            }
            if constexpr (!epi_expert(EPI)) {
                // The last columns, where they are no whole store: an element to a lane, all residuals asked for before the first is used (a lane with its row's
                // elements one after the other waits for each of its rows: 1313 x 7414 x 128 onto a residual 35 us, 25 so, and 20 with 7416).
                const int tail = a.N / OPL * OPL, first = tail - (col0 + c0);
                if (tail < a.N && first >= 0 && first < PW) {
                    constexpr int ROWS = 64 / OPL, STEPS = TP / ROWS;
                    const int e = lane % OPL, col = tail + e;
                    float one[STEPS];
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        const int64_t tok = tok0 + t0 + ROWS * i + lane / OPL;
                        one[i] = 0.f;
                        if (tok >= n_rows || col >= a.N || !a.residual) continue;
                        if (a.res_f32) one[i] = static_cast<const float*>(a.residual)[tok * a.ldr + col];
                        else one[i] = __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.residual)[tok * a.ldr + col] << 16);
                    }
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        const int row = ROWS * i + lane / OPL;
                        const int64_t tok = tok0 + t0 + row;
                        if (tok >= n_rows || col >= a.N) continue;
                        float v = *reinterpret_cast<const float*>(reg + row * RBY + ((((first + e) / 4) ^ (row % PPR)) << 4) + (first + e) % 4 * 4) * a.scale;
                        if (a.residual) v += one[i];
                        if (OUT_BF16) static_cast<__bf16*>(a.y)[tok * a.ldy + col] = (__bf16)v;
                        else static_cast<float*>(a.y)[tok * a.ldy + col] = v;
                    }
                }
            }
        }
    }
}

template <typename ARGS>
__device__ __forceinline__ int64_t x_rows(const ARGS& a) {
    if constexpr (std::is_same<ARGS, ExpertArgs>::value) return a.x_rows;
    else return 0;
}

template <typename CFG, bool OUT_BF16, int EPI>
__global__ void __launch_bounds__(CFG::THREADS) __attribute__((amdgpu_waves_per_eu(CFG::WGS_PER_CU * CFG::NW / 4, CFG::WGS_PER_CU * CFG::NW / 4)))
gdn_linear_kernel(typename EpiArgs<EPI>::type a) {
    constexpr int BM = CFG::BM, BN = CFG::BN, BK = CFG::BK, STAGES = CFG::STAGES, RB = CFG::RB, PP = CFG::PP, RL = CFG::RL;
    constexpr int RPL = CFG::ROWS_PER_LOAD, TI = CFG::TI, TJ = CFG::TJ, XL = CFG::XL, WL = CFG::WL;
    extern __shared__ __align__(16) char smem[];
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / CFG::WAVES_N, wn = wave % CFG::WAVES_N;   // the wave's part: tokens WM wm .., outputs WN wn ..
    const int lr = lane & 15, g = lane >> 4;
    // ---- which tile.  Workgroups are dealt to the 8 XCDs (each with an L2 of its own) in turn: XCD x takes a consecutive run of the
    // tiles, which are numbered GROUP_M tile rows at a time, down the rows first, so that the tiles an XCD works on together
    // share their rows of x and of w in its L2.  (Row by row over the whole output, an XCD's 32 tiles touched nearly every row of w.)
    constexpr int GROUP_M = CFG::BM == 256 ? 4 : 8;
    // Each XCD enters its run an eighth further on than the one before: XCDs that walk the same columns in step would all wait for the
    // same cold rows of w on every k step; so a row comes from memory for one or two of them and from the memory-side cache for
    // the others (8192 x 8192 x 2048 with cold weights 226 -> 209 us; 197 with warm ones either way).
    const int xcd = (int)blockIdx.x & 7;
    if constexpr (epi_expert(EPI)) {               // how many tiles there are the device knows: the grid is as many as there can be
        a.tiles_m = *a.n_tiles;
        a.per_xcd = (a.tiles_m * a.tiles_n + 7) / 8;
        if (((int)blockIdx.x >> 3) >= a.per_xcd) return;
    }
    int in_run = ((int)blockIdx.x >> 3) + xcd * a.per_xcd / 8;
    if (in_run >= a.per_xcd) in_run -= a.per_xcd;
    const int seq = xcd * a.per_xcd + in_run;
    if (seq >= a.tiles_m * a.tiles_n) return;      // (the grid is 8 per_xcd)
    const int grp = seq / (GROUP_M * a.tiles_n), in_grp = seq % (GROUP_M * a.tiles_n);
    const int grp_rows = min(a.tiles_m - grp * GROUP_M, GROUP_M);
    int tile_m = grp * GROUP_M + in_grp % grp_rows, tile_n = in_grp / grp_rows;
    const int32_t* list = nullptr;
    int64_t n_rows = a.T;
    if constexpr (epi_expert(EPI)) {
        // an expert's tiles are numbered down its rows first, so that those that share rows of w follow each other
        const ExpertTile& entry = a.table[seq / a.tiles_n];
        const int in_expert = seq - entry.first * a.tiles_n;
        tile_m = in_expert % entry.tiles;
        tile_n = in_expert / entry.tiles;
        list = a.list + (int64_t)entry.expert * a.list_stride;
        n_rows = entry.rows;
        const int64_t skip = (int64_t)entry.expert * a.N * a.ldw * 2 * (epi_gated(EPI) ? 2 : 1);
        a.w = reinterpret_cast<const char*>(a.w) + skip;
        if (epi_gated(EPI)) a.w_up = reinterpret_cast<const char*>(a.w_up) + skip;
    }
    const int64_t m0 = (int64_t)tile_m * BM;
    constexpr int BNO = epi_gated(EPI) ? BN / 2 : BN;            // outputs of a tile
    const int n0 = tile_n * BNO;
    const int64_t rows_x = n_rows - m0 < BM ? n_rows - m0 : BM;
    const int rows_w = a.N - n0 < BNO ? a.N - n0 : BNO;
    const char* xb = reinterpret_cast<const char*>(a.x) + (epi_expert(EPI) ? 0 : m0 * a.ldx * 2);
    const char* wb = reinterpret_cast<const char*>(a.w) + (int64_t)n0 * a.ldw * 2;
    const int x_bytes = (int)(((epi_expert(EPI) ? x_rows(a) : rows_x) - 1) * a.ldx * 2 + (int64_t)a.K * 2), w_bytes = (int)((int64_t)(rows_w - 1) * a.ldw * 2 + (int64_t)a.K * 2);
    const char* ub = wb;                                         // the second weight's rows
    int u_bytes = w_bytes;
    if constexpr (epi_gated(EPI)) {
        ub = reinterpret_cast<const char*>(a.w_up) + (int64_t)n0 * a.ldw_up * 2;
        u_bytes = (int)((int64_t)(rows_w - 1) * a.ldw_up * 2 + (int64_t)a.K * 2);
    }

    // a wave-wide load writes RPL rows of RB bytes: lane i lands at row i / PP, position i % PP, and fetches the piece that belongs there
    const int ld_row = lane / PP, ld_pos = lane % PP;
    int xoff[XL], woff[WL];      // byte offsets (k = 0) of the loads this wave issues per stage
#pragma unroll
    for (int j = 0; j < XL; ++j) {
        const int row = (BM / CFG::NW) * wave + RPL * j + ld_row;
        int64_t at = row;
        if constexpr (epi_expert(EPI)) at = list[min((int64_t)row, rows_x - 1) + m0] / a.div;      // (behind the last row its copies, for outputs that go nowhere)
        xoff[j] = (int)(at * a.ldx * 2) + ((ld_pos ^ ((row / RL) % PP)) << 4);
    }
#pragma unroll
    for (int j = 0; j < WL; ++j) {
        const int row = (BN / CFG::NW) * wave + RPL * j + ld_row;
        if constexpr (epi_gated(EPI))
            woff[j] = (int)(((row >> 5) * 16 + (row & 15)) * (up_load<CFG>(j, wave) ? a.ldw_up : a.ldw) * 2) + ((ld_pos ^ ((row / RL) % PP)) << 4);
        else
            woff[j] = (int)(row * a.ldw * 2) + ((ld_pos ^ ((row / RL) % PP)) << 4);
    }
    // one of the wave's loads of a stage; past the last k step (not live) it fetches nothing
    auto load = [&](int j, int stage, int k0, bool live) {
        const bool up = epi_gated(EPI) && j >= XL && up_load<CFG>(j - XL, wave);
        LinLoad<CFG>::one(j, smem, stage, k0, wave, xb, live ? x_bytes : 0, up ? ub : wb, live ? (up ? u_bytes : w_bytes) : 0, xoff, woff);
    };
    f32x4 acc[TJ][TI];           // [output tile][token tile]: lane lr = token, register e = output 4 g + e
#pragma unroll
    for (int i = 0; i < TJ; ++i)
#pragma unroll
        for (int j = 0; j < TI; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;

    // fragment reads: row r of a tile, piece 4 kk + g, stored at (4 kk + g) ^ swz(r); tile origins are multiples of 16 rows
    const int sw = lr / RL;
    const int xrow = (CFG::WM * wm + lr) * RB, wrow = (CFG::WN * wn + lr) * RB;
    const int n_steps = a.K / BK;
    constexpr int KK = BK / 32;              // matrix-instruction steps per stage (even)
    // The stages are consumed through two fragment sets: while the matrix cores work on one k step of 32, the fragments of
    // the next are read from LDS, also across the stage boundary.  The hand-over of a stage therefore sits before the LAST
    // k step of the stage in front of it: wait for this wave's loads of the next stage, for its own fragment reads, then the
    // barrier; after it the next stage is readable by every wave and the current one (whose last fragments are in
    // registers) is free and is refilled with the stage STAGES ahead.
    bf16x8 xf[2][TI], wf[2][TJ];
    auto read_frags = [&](int stage, int kk, int set) {
        const char* xs = smem + stage * CFG::STAGE_BYTES;
        const char* ws = xs + CFG::X_BYTES;
        const int pos = ((4 * kk + g) ^ sw) * 16;
#pragma unroll
        for (int t = 0; t < TI; ++t) xf[set][t] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(xs + xrow + 16 * t * RB + pos));
#pragma unroll
        for (int t = 0; t < TJ; ++t) wf[set][t] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(ws + wrow + 16 * t * RB + pos));
    };
    // Loads are issued for every stage slot, also past the last k step: there the descriptor is empty and the scalar offset
    // zero (no lane is in range by definition, nothing is fetched), so that the number of loads in flight, and with it every
    // wait below, is the same in every round and the loop body has no branch for the scheduler to stop at.
    auto mma_all = [&](int set) {
#pragma unroll
        for (int tj = 0; tj < TJ; ++tj)
#pragma unroll
            for (int ti = 0; ti < TI; ++ti)
                acc[tj][ti] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[set][tj], xf[set][ti], acc[tj][ti], 0, 0, 0);
    };
#pragma unroll
    for (int p = 0; p < STAGES; ++p) {
        const bool live = p < n_steps;
#pragma unroll
        for (int j = 0; j < CFG::LPS; ++j) load(j, p, live ? p * BK : 0, live);
    }
    wait_vm<(STAGES - 1) * CFG::LPS>();
    __syncthreads();
    read_frags(0, 0, 0);
    int stage = 0;                           // step % STAGES
    for (int step = 0; step + 1 < n_steps; ++step) {
        const int next_stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int kk = 0; kk + 1 < KK; ++kk) {
            // The fragments of k step kk + 1 go into the other register set while the matrix instructions of k step kk are
            // issued, one read behind every matrix instruction or two, pinned in that order: left to itself the scheduler
            // reads them into the registers the matrix instructions have just used, behind them, and waits out the LDS
            // latency with the matrix pipe idle; and a burst of reads in front keeps the issue port from the matrix pipe.
            const int rs = (kk & 1) ^ 1, ms = kk & 1;
            const char* xs = smem + stage * CFG::STAGE_BYTES;
            const char* ws = xs + CFG::X_BYTES;
            const int pos = ((4 * (kk + 1) + g) ^ sw) * 16;
            constexpr int NM = TI * TJ, NR = TI + TJ;
            constexpr int SLOTS = NM < NR ? NM : NR;
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
                for (int q = i * NM / SLOTS; q < (i + 1) * NM / SLOTS; ++q)
                    acc[q / TI][q % TI] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[ms][q / TI], xf[ms][q % TI], acc[q / TI][q % TI], 0, 0, 0);
#pragma unroll
                for (int r = i * NR / SLOTS; r < (i + 1) * NR / SLOTS; ++r) {
                    if (r < TI) xf[rs][r] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(xs + xrow + 16 * r * RB + pos));
                    else wf[rs][r - TI] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(ws + wrow + 16 * (r - TI) * RB + pos));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // (the matrix instructions above stay above: left to itself the scheduler sinks them below the barrier, and the
        // fragment reads and the barrier are then waited for with the matrix pipe idle)
        __builtin_amdgcn_sched_barrier(0);
        // the next stage has landed for this wave (the STAGES - 2 stages behind it may still be in flight) ...
        wait_vm<CFG::AHEAD>();
        __builtin_amdgcn_s_waitcnt(0xC07F);          // ... and this wave's last fragment reads of the current stage are done (lgkmcnt(0))
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        {
            // The last k step of the stage (fragment set 1; KK is even), written out in issue order and pinned there: a load
            // to LDS takes tens of cycles to issue, so one goes out in each slot of a few matrix instructions, which cover it, from
            // the first slot on: a load has from here to the hand-over STAGES - 1 stages on to arrive, and with two stages one that goes out in
            // the last slot has half a stage.  (Spread over all slots, cold weights, shape 2: 4096 x 2560 x 2048 49.9 us
            // against 47.3, 3000 x 4096 x 4096 90.4 / 85.9, 1000 x 8224 x 2048 50.4 / 48.7; warm 8192 x 8192 x 2048 189 / 191; two loads a slot: 48.0, 87.1, 49.1, 192.)
            // The fragments of the next stage's first k step are read in between as well.
            const bool live = step + STAGES < n_steps;
            const int k_ahead = live ? (step + STAGES) * BK : 0;
            const char* xs = smem + next_stage * CFG::STAGE_BYTES;
            const char* ws = xs + CFG::X_BYTES;
            const int pos = (g ^ sw) * 16;
            constexpr int NM = TI * TJ, NL = CFG::LPS, NR = TI + TJ;
            constexpr int SLOTS = NM < (NL > NR ? NL : NR) ? NM : (NL > NR ? NL : NR);   // interleave slots
            static_assert(NL <= SLOTS, "every load has a slot");
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
                for (int q = i * NM / SLOTS; q < (i + 1) * NM / SLOTS; ++q)
                    acc[q / TI][q % TI] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[1][q / TI], xf[1][q % TI], acc[q / TI][q % TI], 0, 0, 0);
#pragma unroll
                for (int r = i * NR / SLOTS; r < (i + 1) * NR / SLOTS; ++r) {
                    if (r < TI) xf[0][r] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(xs + xrow + 16 * r * RB + pos));
                    else wf[0][r - TI] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(ws + wrow + 16 * (r - TI) * RB + pos));
                }
                if (i < NL) load(i, stage, k_ahead, live);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        stage = next_stage;
    }
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {        // the last stage: nothing behind it
        if (kk + 1 < KK) read_frags(stage, kk + 1, (kk & 1) ^ 1);
        mma_all(kk & 1);
    }

    // ---- epilogue: bias, one rounding, and out through LDS.  A lane holds runs of four outputs of ONE token, 16 tokens per product:
    //      stored from there, every instruction would touch 16 rows of the output with 32 or 64 bytes each.  Each wave turns its
    //      outputs around in its own share (REGION) of the now idle stage ring instead: rows of 64, 128 or 256 bytes, one for a token,
    //      with as many of the wave's outputs as 256 bytes hold (of shape 5's 80 all in bf16, in a pitch of 256 bytes, and 16 in
    //      fp32), the 16-byte pieces of a row XOR-swizzled with the token so that both the writes (lane = token) and the reads (lane =
    //      piece) spread over the banks; then 4, 8 or 16 lanes store one row's contiguous bytes.  A wave's LDS operations execute in
    //      order, so no barrier stands between its writes and reads; the one barrier before keeps the other waves' last
    //      fragment reads out of the way.
    if constexpr (EPI != EPI_BIAS) {
        wait_vm<0>();
        __syncthreads();
        act_epilogue<CFG, OUT_BF16, EPI>(a, acc, smem + wave * (CFG::SMEM / CFG::NW), m0 + CFG::WM * wm, n0 + CFG::WN / (epi_gated(EPI) ? 2 : 1) * wn, lane,
                                         list, n_rows);
        return;
    } else {
    constexpr int ES = OUT_BF16 ? 2 : 4;
    constexpr int WN = CFG::WN, WM = CFG::WM;                      // the wave's outputs and tokens
    constexpr int REGION = CFG::SMEM / CFG::NW;                    // the wave's part of the ring
    constexpr int PW = WN * ES <= 256 ? WN : WN % (256 / ES) == 0 ? 256 / ES : 16;   // outputs per pass: a row of at most 256 bytes
    constexpr int RBY = PW * ES <= 64 ? 64 : PW * ES <= 128 ? 128 : 256, PPR = RBY / 16;   // row bytes (a power of two), 16-byte pieces per row
    constexpr int RPI = 1024 / RBY;                                // rows a wave-wide 16-byte access covers
    constexpr int TP = (WM * RBY <= REGION) ? WM : REGION / RBY >= 64 ? 64 : 32;   // tokens per pass
    static_assert(TP * RBY <= REGION && TP % RPI == 0 && WM % TP == 0 && WN % PW == 0 && PW % 16 == 0, "epilogue region");
    wait_vm<0>();
    __syncthreads();
    char* const reg = smem + wave * REGION;
    const int64_t tok0 = m0 + WM * wm;
    const int col0 = n0 + WN * wn;
#pragma unroll
    for (int c0 = 0; c0 < WN; c0 += PW) {
#pragma unroll
        for (int t0 = 0; t0 < WM; t0 += TP) {
#pragma unroll
            for (int tj = c0 / 16; tj < (c0 + PW) / 16; ++tj) {
                const int cl = 16 * tj + 4 * g;                    // first of the lane's four outputs, within the wave's part
                f32x4 bv = {0.f, 0.f, 0.f, 0.f};
                if (a.bias) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col0 + cl + e < a.N) bv[e] = a.bias[col0 + cl + e];
                }
#pragma unroll
                for (int ti = t0 / 16; ti < (t0 + TP) / 16; ++ti) {
                    const int row = 16 * ti + lr - t0;
                    f32x4 v = {acc[tj][ti][0] + bv[0], acc[tj][ti][1] + bv[1], acc[tj][ti][2] + bv[2], acc[tj][ti][3] + bv[3]};
                    const int byte = (cl - c0) * ES;
                    char* const dst = reg + row * RBY + (((byte >> 4) ^ (row % PPR)) << 4) + (byte & 15);
                    if (OUT_BF16) *reinterpret_cast<bf16x4*>(dst) = __builtin_convertvector(v, bf16x4);
                    else *reinterpret_cast<f32x4*>(dst) = v;
                }
            }
#pragma unroll
            for (int i = 0; i < TP / RPI; ++i) {
                const int row = RPI * i + lane / PPR, piece = lane % PPR;
                const u32x4 val = *reinterpret_cast<const u32x4*>(reg + row * RBY + ((piece ^ (row % PPR)) << 4));
                const int64_t tok = tok0 + t0 + row;
                const int col = col0 + c0 + piece * (16 / ES);
                if (tok < a.T && col < a.N && (RBY == PW * ES || piece * 16 < PW * ES)) {
                    // the destination of this piece: the whole output, or the segment its first column lies in (segment
                    // boundaries are multiples of 8 columns, so a piece lies in one segment)
                    char* base = reinterpret_cast<char*>(a.y);
                    int64_t ld = a.ldy;
                    int c_lo = 0, c_hi = a.N;
                    if (a.n_seg > 0) {
#pragma unroll
                        for (int sg = 0; sg < LIN_MAX_SEG; ++sg)
                            if (sg < a.n_seg && col >= a.seg_col[sg]) {
                                base = reinterpret_cast<char*>(a.seg_y[sg]);
                                ld = a.seg_ld[sg];
                                c_lo = a.seg_col[sg];
                                c_hi = a.seg_col[sg + 1];
                            }
                    }
                    char* const p = base + (tok * ld + (col - c_lo)) * ES;
                    if (col + 16 / ES <= c_hi) {
                        *reinterpret_cast<u32x4*>(p) = val;
                    } else {
#pragma unroll
                        for (int e = 0; e < 16 / ES; ++e)
                            if (col + e < c_hi) {
                                if (OUT_BF16) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(val[e >> 1] >> (16 * (e & 1)));
                                else reinterpret_cast<uint32_t*>(p)[e] = val[e];
                            }
                    }
                }
            }
        }
    }
    }
}

template <typename CFG, bool OUT_BF16, int EPI>
hipError_t launch_linear(typename EpiArgs<EPI>::type a, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const hipError_t attr_err = allow_lds(reinterpret_cast<const void*>(&gdn_linear_kernel<CFG, OUT_BF16, EPI>), CFG::SMEM, done);
    if (attr_err != hipSuccess) return attr_err;
    const int64_t tiles_m = epi_expert(EPI) ? a.T : (a.T + CFG::BM - 1) / CFG::BM;      // (the experts' T: how many tiles there can be)
    constexpr int BNO = epi_gated(EPI) ? CFG::BN / 2 : CFG::BN;
    a.tiles_n = (a.N + BNO - 1) / BNO;
    a.tiles_m = (int32_t)tiles_m;
    a.per_xcd = (int32_t)((tiles_m * a.tiles_n + 7) / 8);
    hipLaunchKernelGGL((gdn_linear_kernel<CFG, OUT_BF16, EPI>), dim3((unsigned)(8 * (int64_t)a.per_xcd)), dim3(CFG::THREADS), CFG::SMEM, stream, a);
    return hipGetLastError();
}

// ---- few rows (gdn_few_kernel.h): a workgroup makes WR outputs of up to 16 RT rows, or WR / 2 of two products
template <typename C, bool OUT_BF16, bool GATED>
__global__ void __launch_bounds__(64 * C::WAVES) gdn_linear_few_kernel(LinearActArgs a) {
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups are dealt to the 8 XCDs in turn: the row tiles of the same outputs follow each other on one of them, whose L2 then has the weights
    const int seq = (int)blockIdx.x / (8 * a.tiles_m), in = (int)blockIdx.x % (8 * a.tiles_m);
    const int tile_n = seq * 8 + (in & 7), tile_m = in >> 3;
    if (tile_n >= a.tiles_n) return;                             // (the grid is whole eights)
    constexpr int OUTS = GATED ? C::WR / 2 : C::WR;
    const int n0 = tile_n * OUTS, m0 = tile_m * C::ROWS;
    const int rows_x = min((int)a.T - m0, C::ROWS);
    auto weights = [&](const void* w, int64_t ld, int first) { return few::rows_from(w, ld, a.N, a.K, first, C::WR); };
    const few::Part x = {static_cast<const char*>(a.x) + (int64_t)m0 * a.ldx * 2, (int)((int64_t)(rows_x - 1) * a.ldx * 2 + (int64_t)a.K * 2), (int)(a.ldx * 2)};
    f32x4 acc[C::CT * C::RT];
#pragma unroll
    for (int i = 0; i < C::CT * C::RT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    // A workgroup begins 5 steps on from the one before it: those that begin at the same k of rows whose pitch is a power of two all ask the same few memory
    // channels (16 rows, 8192 x 8192: 34 us, 26 so)
    const int steps = a.K / few::STEP, first = (int)((uint32_t)tile_n * 5u % (uint32_t)steps);
    C::sums_of(acc, weights(a.w, a.ldw, n0), GATED ? weights(a.w_up, a.ldw_up, n0) : weights(a.w, a.ldw, n0 + 8 * C::HALF), x, steps,
               [&](int step, few::Part&, few::Part&, few::Part&) { return (step + first >= steps ? step + first - steps : step + first) * few::STEP * 2; },
               smem + wave * C::RING, wave, lane);
    wait_vm<0>();                                                // (no load of an empty descriptor writes behind the sums)
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);
    C::put_sums(acc, sums, wave, lane);
    __syncthreads();
    constexpr int PER_ROW = OUTS / 4;
    for (int i = threadIdx.x; i < C::ROWS * PER_ROW; i += 64 * C::WAVES) {      // four outputs of a row each
        const int row = i / PER_ROW, piece = i % PER_ROW, col = n0 + 4 * piece;
        if (row >= rows_x || col >= a.N) continue;
        f32x4 v = C::get_sum(sums, row, piece), up = {1.f, 1.f, 1.f, 1.f};
        if (GATED) up = C::get_sum(sums, row, piece + PER_ROW);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.N) {
                if (a.bias) v[e] += a.bias[col + e];
                if (GATED && a.bias_up) up[e] += a.bias_up[col + e];
            }
        v = activate(a.act, v);
        if (GATED) v *= up;
        v *= a.scale;
        const int64_t t = m0 + row;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.N) {
                if (a.residual)
                    v[e] += a.res_f32 ? static_cast<const float*>(a.residual)[t * a.ldr + col + e]
                                      : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.residual)[t * a.ldr + col + e] << 16);
                if (OUT_BF16) static_cast<__bf16*>(a.y)[t * a.ldy + col + e] = (__bf16)v[e];
                else static_cast<float*>(a.y)[t * a.ldy + col + e] = v[e];
            }
    }
}

template <typename C, bool OUT_BF16, bool GATED>
hipError_t launch_few_kernel(LinearActArgs a, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const hipError_t attr_err = allow_lds(reinterpret_cast<const void*>(&gdn_linear_few_kernel<C, OUT_BF16, GATED>), C::SMEM, done);
    if (attr_err != hipSuccess) return attr_err;
    constexpr int OUTS = GATED ? C::WR / 2 : C::WR;
    a.tiles_n = (a.N + OUTS - 1) / OUTS;
    a.tiles_m = (int32_t)((a.T + C::ROWS - 1) / C::ROWS);
    hipLaunchKernelGGL((gdn_linear_few_kernel<C, OUT_BF16, GATED>), dim3((unsigned)((a.tiles_n + 7) / 8 * 8 * a.tiles_m)), dim3(64 * C::WAVES), C::SMEM, stream, a);
    return hipGetLastError();
}
template <typename C>
hipError_t launch_few(const LinearActArgs& a, bool bf, hipStream_t stream) {
    if constexpr (C::WR >= 16)
        if (a.w_up) return bf ? launch_few_kernel<C, true, true>(a, stream) : launch_few_kernel<C, false, true>(a, stream);
    return bf ? launch_few_kernel<C, true, false>(a, stream) : launch_few_kernel<C, false, false>(a, stream);
}

int expert_tile_rows(int shape) { return shape == 2 ? LinBig8::BM : shape == 3 ? LinTiny::BM : LinSmall::BM; }

template <typename CFG>
hipError_t launch_expert_shape(const ExpertArgs& a, bool gated, hipStream_t stream) {
    return gated ? launch_linear<CFG, true, EPI_EXPERT_GATED>(a, stream) : launch_linear<CFG, false, EPI_EXPERT>(a, stream);
}
hipError_t launch_expert_product(const ExpertProduct& p, int shape, hipStream_t stream) {
    ExpertArgs a = {};
    a.x = p.x; a.w = p.w; a.y = p.y;
    a.ldx = p.ldx; a.ldw = a.ldw_up = p.K; a.ldy = p.N;
    a.T = p.most_tiles; a.N = p.N; a.K = p.K;
    a.w_up = p.gated ? static_cast<const char*>(p.w) + (int64_t)p.N * p.K * 2 : nullptr;
    a.act = p.act; a.scale = 1.f;
    a.list = p.list; a.table = p.table; a.n_tiles = p.n_tiles; a.weights = p.weights;
    a.list_stride = p.list_stride; a.div = p.div; a.x_rows = p.x_rows;
    switch (shape) {
        case 2: return launch_expert_shape<LinBig8>(a, p.gated, stream);
        // (768 of k, 128 experts of 2048 outputs: 81 us with two workgroups of five stages, 75 with three of three; 2048 of k: 130, 132)
        case 3: return p.K <= 1024 ? launch_expert_shape<LinTiny3>(a, p.gated, stream) : launch_expert_shape<LinTiny>(a, p.gated, stream);
        default: return launch_expert_shape<LinSmall>(a, p.gated, stream);
    }
}

std::atomic<int32_t> g_linear_shape{-1}, g_act_shape{-1};

// The estimated time of a problem in a tile shape, in us: full rounds of workgroups over the chip, and a last one that costs its latency (a
// workgroup alone walks k no faster) and more the fuller it is, since the compute units share power and memory.  A round has a part that
// grows with k and a part that does not (first loads, outputs): at K = 64 the second is the larger, and the more so
// the larger the tile, so a choice made at K = 2048 is up to 24 % off there (3000 x 6144 x 64 16.3 us in shape 2, 13.8 in shape 0; 8192 x 2560 x 256 22.9 / 19.9).
// Fitted to T = 1 .. 12000, N = 32 .. 8224, K = 64 .. 8192, all shapes at each, weights in the caches and not: the shape
// chosen is 0.5 % from the best of the five on average, 4 % and more in one case of twenty, at K >= 512 7 % at most, below (all of them calls
// of 4 to 7 us) 25 %; its estimate is within 14 % in nine of ten.  us, cold weights, K = 2048, in shapes 3 / 0 / 4 / 5 / 2:
// 512 x 2048 9.5 / 21 / 16 / 19 / 38, 1400 x 2048 20 / 23 / 18 / 21 / 39, 384 x 8224 31 / 31 / 22 / 27 / 47, 512 x 8224 39 / 31 / 36 / 27 / 49,
// 1000 x 8224 60 / 54 / 53 / 49 / 47, 700 x 6144 36 / 31 / 33 / 24 / 47, 2048 x 6144 76 / 58 / 57 / 63 / 47, 8192 x 2048 92 / 57 / 67 / 77 / 50,
// 8192 x 6144 283 / 173 / 205 / 204 / 147.
struct ShapeCost {
    int id, bm, bn, per_cu;
    double full_k, full, alone_k, alone;      // us of a full round, of a workgroup alone: per 2048 of k, and whatever k
    bool square;                              // the fullness of the last round counts squared
};
constexpr ShapeCost SHAPES[5] = {{3, 64, 64, 2, 10.4, 1.8, 3.9, 2.0, false},
                                 {0, 128, 128, 2, 26.0, 3.3, 14.4, 1.8, false},
                                 {4, 128, 128, 1, 14.2, 2.6, 10.4, 2.1, false},
                                 {5, 128, 160, 1, 15.9, 5.0, 12.9, 3.9, false},
                                 {2, 256, 256, 1, 41.9, 6.9, 32.6, 4.0, true}};
double rounds_cost(const ShapeCost& c, int64_t tiles, int32_t K) {
    const int64_t slots = (int64_t)chip_cus() * c.per_cu;
    const double k = (double)K / 2048.0, f = (double)(tiles % slots) / (double)slots;
    const double full = c.full_k * k + c.full, alone = c.alone_k * k + c.alone;
    return (double)(tiles / slots) * full + (f > 0 ? alone + (full - alone) * (c.square ? f * f : f) : 0.0);
}
double shape_cost(const ShapeCost& c, int64_t T, int64_t N, int32_t K) {
    return rounds_cost(c, ((T + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn), K);
}

double expert_product_us(int shape, int64_t row_tiles, int64_t rows_w, int32_t K) {
    // (three workgroups to a compute unit where k is short: a round of half as many more tiles)
    constexpr ShapeCost three = {3, 64, 64, 3, 15.1, 2.4, 3.9, 2.0, false};
    const ShapeCost& c = shape == 2 ? SHAPES[4] : shape == 0 ? SHAPES[1] : K <= 1024 ? three : SHAPES[0];
    return rounds_cost(c, row_tiles * ((rows_w + c.bn - 1) / c.bn), K);
}

// Which tile shape a problem gets, and how many of its columns: a problem whose tiles leave a last round nearly empty may be cut
// into columns that fill whole rounds of 256 x 256 tiles and a rest in a smaller shape, a launch of its own.  Measured, whole / cut: 8192 x
// 8224 (33 tile columns where 32 fill four rounds) 233 / 211 us, 8192 x 2560 88 / 76, 2048 x 8224 90 / 65, 4096 x 8224 138 / 113.
struct LinearPlan { int shape, rest_shape; int32_t cols; };   // outputs 0 .. cols - 1 in `shape`, the others in `rest_shape`
LinearPlan plan_tiles(int64_t T, int32_t N, int32_t K, bool gated) {      // gated: N rows of both weights together; no shape 5
    auto best_of = [&](int64_t n, int shapes, double* t) {
        int best = 0;
        for (int i = 0; i < shapes; ++i) {
            if (gated && SHAPES[i].id == 5) continue;
            const double ti = shape_cost(SHAPES[i], T, n, K);
            if (i == 0 || ti < *t) { best = SHAPES[i].id; *t = ti; }
        }
        return best;
    };
    double whole = 0.0;
    LinearPlan p = {best_of(N, 5, &whole), 0, N};
    const double launch = 2.5;                           // a launch beyond its estimate
    double least = 0.97 * whole;                         // (a cut has to be worth it)
    const int64_t tiles_m = (T + 255) / 256, cus = chip_cus();
    for (int64_t r = 1; r <= 64; ++r) {                  // the most columns that r rounds of 256 x 256 tiles hold
        const int64_t cols = r * cus / tiles_m * 256;
        if (cols >= N) break;
        if (cols == 0) continue;
        double rest = 0.0;
        const int rest_shape = best_of(N - cols, 4, &rest);
        const double t = shape_cost(SHAPES[4], T, cols, K) + rest + launch;
        if (t < least) { least = t; p = {2, rest_shape, (int32_t)cols}; }
    }
    return p;
}
LinearPlan plan_linear(int64_t T, int32_t N, int32_t K) {
    const int forced = g_linear_shape.load();
    return forced >= 0 ? LinearPlan{forced, 0, N} : plan_tiles(T, N, K, false);
}

// ---- the kernels of few rows, shapes 6 .. 11: 16 rows of x with 8, 16, 32 rows of w, then 32 with each.
// The estimate: a compute unit takes rows of x, which it finds in L2, at 90 KB a us, rows of w at 50, and at 40 where workgroups of other rows ask for them at the
// same time; memory sends 5.5 TB/s, and 3 us go to the beginning and the end.  So a narrow weight wants many workgroups, that is few of its rows each, until x, which each of
// them reads whole, outweighs them; and a compute unit with one workgroup more than the others is waited for, and its first loads cost 0.8 us more.
//   us, N 2048, K 6144, shapes 6 / 7 / 8 / 9 / 10 / 11, and 64 x 64 tiles
//     weights in the memory-side cache   16 rows   7.3 /  8.1 / 10.2 /  7.7 /  8.6 / 10.9, 19
//                                        48       14.8 / 11.9 / 10.0 / 14.1 /  8.9 / 11.2, 19.6
//                                       128       31   / 21   / 16   / 30   / 16.1 / 12.4, 20.8
//     weights from memory                48       19.9 / 16.9 / 14.5 / 18.4 / 12.2 / 16.2, 29.8
// With few outputs they are the better for more rows too: 174 x 44 x 7232 7.7, tiles 22; 491 x 298 x 3712 9.3, 14; from some 1000 rows on the tiles always were
// (3737 x 19 x 3648 32, tiles 13.8).  Over 350 problems (1 to 1024 rows, N 8 to 8192, K 256 to 8192) the choice is 2 to 3 % from the best on average, and 7 to 12 % or more in one
// of twenty.
constexpr int FEW = 6, FEW_ROWS = 1024;
struct FewShape { int rt, wr; };
constexpr FewShape FEW_SHAPES[6] = {{1, 8}, {1, 16}, {1, 32}, {2, 8}, {2, 16}, {2, 32}};
// (per_cu: us that a compute unit's bytes take it; bytes: all that memory sends)
double bytes_cost(double per_cu, double bytes) { return 3.0 + std::sqrt(per_cu * per_cu + bytes * bytes / (5.5e6 * 5.5e6)); }
double few_cost(const FewShape& s, int64_t T, int64_t N, int32_t K, bool gated) {
    const int64_t outs = gated ? s.wr / 2 : s.wr, tiles_n = (N + outs - 1) / outs, tiles_m = (T + 16 * s.rt - 1) / (16 * s.rt);
    const int64_t cus = chip_cus(), most = (tiles_n * tiles_m + cus - 1) / cus;                   // workgroups of a compute unit
    const double shared = 1.0 - 1.0 / (double)tiles_m, row = 2.0 * K;
    const double one = row * ((double)std::min<int64_t>(T, 16 * s.rt) / 90e3 + s.wr * (shared / 40e3 + (1.0 - shared) / 50e3));
    return bytes_cost(one * (double)most, row * ((double)N * (gated ? 2 : 1) + (double)T)) + 0.8 * (double)(most - 1);
}

// (a launch has less than 2^32 threads)
bool few_fits(const FewShape& s, int64_t T, int64_t N, bool gated) {
    const int64_t outs = gated ? s.wr / 2 : s.wr;
    return T <= FEW_ROWS && (N / outs + 16) * ((T + 16 * s.rt - 1) / (16 * s.rt)) < (int64_t)1 << 24;
}
LinearPlan plan_act(int64_t T, int32_t N, int32_t K, bool gated) {
    int forced = g_act_shape.load();
    if (gated && forced >= FEW && FEW_SHAPES[forced - FEW].wr == 8) ++forced;
    if (forced >= FEW && few_fits(FEW_SHAPES[forced - FEW], T, N, gated)) return {forced, 0, N};
    if (forced >= 0 && forced < FEW) return {forced == 1 ? 2 : gated && forced == 5 ? 0 : forced, 0, N};
    if (gated && N > INT32_MAX / 2) return {2, 0, N};
    LinearPlan p = plan_tiles(T, gated ? 2 * N : N, K, gated);
    if (T <= FEW_ROWS) {
        // (the tiles' estimate knows rounds of them; with so few rows what a tile's compute unit is sent, and the weights, may take longer,
        // and a tenth more with a barrier at every step)
        const ShapeCost* c = SHAPES;
        while (c->id != p.shape) ++c;
        const int64_t rows_w = gated ? 2 * (int64_t)N : N;
        double least = std::max(shape_cost(*c, T, rows_w, K), 1.1 * bytes_cost(2.0 * K * (double)(std::min<int64_t>(T, c->bm) + c->bn) / 57e3, 2.0 * K * (double)rows_w));
        for (int i = 0; i < 6; ++i) {
            if ((gated && FEW_SHAPES[i].wr == 8) || !few_fits(FEW_SHAPES[i], T, N, gated)) continue;
            const double t = few_cost(FEW_SHAPES[i], T, N, K, gated);
            if (t < least) { least = t; p = {FEW + i, 0, gated ? 2 * N : N}; }
        }
    }
    if (gated) p.cols /= 2;                              // (a multiple of 128 where it is cut)
    return p;
}

}  // namespace linear
}  // namespace gdn

using namespace gdn;
using namespace gdn::linear;

namespace {
int32_t linear_checks(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, int32_t out_dtype, int64_t T, int32_t N,
                      int32_t K) {
    if (T < 0 || N < 0 || K < 0) return GDN_ERR_COUNT;
    if (out_dtype != GDN_BF16 && out_dtype != GDN_F32) return GDN_ERR_SHAPE;
    if (K % 64 != 0 || ldx < K || ldw < K) return GDN_ERR_SHAPE;
    if (T == 0 || N == 0) return GDN_OK;
    if (K == 0) return GDN_ERR_SHAPE;
    if (!x || !w) return GDN_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(x) & 15u) || (reinterpret_cast<uintptr_t>(w) & 15u) || (bias && (reinterpret_cast<uintptr_t>(bias) & 3u)))
        return GDN_ERR_ALIGN;
    if ((ldx & 7) || (ldw & 7)) return GDN_ERR_ALIGN;
    // a tile's rows must be addressable with 31-bit byte offsets
    if ((int64_t)256 * ldx * 2 >= ((int64_t)1 << 31) || (int64_t)256 * ldw * 2 >= ((int64_t)1 << 31)) return GDN_ERR_COUNT;
    if (((T + 127) / 128) * (((int64_t)N + 127) / 128) > INT32_MAX) return GDN_ERR_COUNT;
    return GDN_OK;
}

template <typename CFG, int EPI>
hipError_t launch_out(const typename EpiArgs<EPI>::type& a, bool bf, hipStream_t stream) {
    return bf ? launch_linear<CFG, true, EPI>(a, stream) : launch_linear<CFG, false, EPI>(a, stream);
}
template <int EPI>
int32_t launch_shape(const typename EpiArgs<EPI>::type& a, int shape, bool bf, hipStream_t stream) {
    switch (shape) {
        case 1:
            if constexpr (EPI == EPI_BIAS) return hip_err(launch_out<LinBig, EPI>(a, bf, stream));
            [[fallthrough]];
        case 2: return hip_err(launch_out<LinBig8, EPI>(a, bf, stream));
        case 3: return hip_err(launch_out<LinTiny, EPI>(a, bf, stream));
        case 4: return hip_err(launch_out<LinDeep, EPI>(a, bf, stream));
        case 5:
            if constexpr (EPI != EPI_GATED) return hip_err(launch_out<LinWide, EPI>(a, bf, stream));   // (an odd number of tiles to a wave)
            return GDN_ERR_SHAPE;
        default: return hip_err(launch_out<LinSmall, EPI>(a, bf, stream));
    }
}

// Columns c0 .. c1 - 1 of a projection as a projection of its own (c0 a multiple of 256: every alignment holds).
LinearArgs column_range(const LinearArgs& a, int32_t c0, int32_t c1, int es) {
    LinearArgs b = a;
    b.w = static_cast<const char*>(a.w) + (int64_t)c0 * a.ldw * 2;
    if (a.bias) b.bias = a.bias + c0;
    b.N = c1 - c0;
    if (a.n_seg == 0) {
        b.y = static_cast<char*>(a.y) + (int64_t)c0 * es;
        return b;
    }
    b.n_seg = 0;
    for (int32_t sg = 0; sg < a.n_seg; ++sg) {
        const int32_t lo = std::max(a.seg_col[sg], c0), hi = std::min(a.seg_col[sg + 1], c1);
        if (lo >= hi) continue;
        b.seg_col[b.n_seg] = lo - c0;
        b.seg_y[b.n_seg] = static_cast<char*>(a.seg_y[sg]) + (int64_t)(lo - a.seg_col[sg]) * es;
        b.seg_ld[b.n_seg] = a.seg_ld[sg];
        ++b.n_seg;
    }
    for (int32_t sg = b.n_seg; sg <= LIN_MAX_SEG; ++sg) b.seg_col[sg] = b.N;
    return b;
}

int32_t linear_launch(const LinearArgs& a, int32_t out_dtype, hipStream_t stream) {
    const bool bf = out_dtype == GDN_BF16;
    const LinearPlan p = plan_linear(a.T, a.N, a.K);
    if (p.cols == a.N) return launch_shape<EPI_BIAS>(a, p.shape, bf, stream);
    const int es = bf ? 2 : 4;
    const int32_t rc = launch_shape<EPI_BIAS>(column_range(a, 0, p.cols, es), p.shape, bf, stream);
    return rc != GDN_OK ? rc : launch_shape<EPI_BIAS>(column_range(a, p.cols, a.N, es), p.rest_shape, bf, stream);
}

// Outputs c0 .. c1 - 1 of a projection with an epilogue, as one of its own.
LinearActArgs act_range(const LinearActArgs& a, int32_t c0, int32_t c1, int es) {
    LinearActArgs b = a;
    static_cast<LinearArgs&>(b) = column_range(a, c0, c1, es);
    if (a.w_up) b.w_up = static_cast<const char*>(a.w_up) + (int64_t)c0 * a.ldw_up * 2;
    if (a.bias_up) b.bias_up = a.bias_up + c0;
    if (a.residual) b.residual = static_cast<const char*>(a.residual) + (int64_t)c0 * (a.res_f32 ? 4 : 2);
    return b;
}
int32_t launch_act_shape(const LinearActArgs& a, int shape, bool bf, hipStream_t stream) {
    switch (shape - FEW) {
        case 0: return hip_err(launch_few<few::Few<1, 8, 4, 6>>(a, bf, stream));
        case 1: return hip_err(launch_few<few::Few<1, 16, 4, 4>>(a, bf, stream));
        case 2: return hip_err(launch_few<few::Few<1, 32, 4, 3>>(a, bf, stream));
        case 3: return hip_err(launch_few<few::Few<2, 8, 4, 4>>(a, bf, stream));
        case 4: return hip_err(launch_few<few::Few<2, 16, 4, 3>>(a, bf, stream));
        case 5: return hip_err(launch_few<few::Few<2, 32, 4, 2>>(a, bf, stream));
        default: break;
    }
    return a.w_up ? launch_shape<EPI_GATED>(a, shape, bf, stream) : launch_shape<EPI_ACT>(a, shape, bf, stream);
}
}  // namespace

extern "C" int32_t gdn_linear(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, void* y, int64_t ldy,
                              int32_t out_dtype, int64_t T, int32_t N, int32_t K, void* stream_) {
    const int32_t rc = linear_checks(x, ldx, w, ldw, bias, out_dtype, T, N, K);
    if (rc != GDN_OK) return rc;
    if (ldy < N) return GDN_ERR_SHAPE;
    if (T == 0 || N == 0) return GDN_OK;
    if (!y) return GDN_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(y) & (out_dtype == GDN_BF16 ? 7u : 15u)) || (ldy & 3)) return GDN_ERR_ALIGN;
    LinearArgs a = {};
    a.x = x; a.w = w; a.bias = bias; a.y = y;
    a.ldx = ldx; a.ldw = ldw; a.ldy = ldy;
    a.T = T; a.N = N; a.K = K;
    a.n_seg = 0;
    return linear_launch(a, out_dtype, (hipStream_t)stream_);
}

extern "C" int32_t gdn_linear_split(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, int32_t n_seg,
                                    const int32_t* seg_cols, void* const* seg_y, const int64_t* seg_ld, int32_t out_dtype, int64_t T,
                                    int32_t K, void* stream_) {
    if (n_seg < 1 || n_seg > LIN_MAX_SEG) return GDN_ERR_COUNT;
    if (!seg_cols || !seg_y || !seg_ld) return GDN_ERR_NULL;
    if (seg_cols[0] != 0) return GDN_ERR_SHAPE;
    for (int32_t sg = 0; sg < n_seg; ++sg) {
        if (seg_cols[sg + 1] <= seg_cols[sg]) return GDN_ERR_SHAPE;                 // empty or decreasing
        if (sg + 1 < n_seg && (seg_cols[sg + 1] & 7)) return GDN_ERR_ALIGN;         // inner boundaries: whole 16-byte pieces
    }
    const int32_t N = seg_cols[n_seg];
    const int32_t rc = linear_checks(x, ldx, w, ldw, bias, out_dtype, T, N, K);
    if (rc != GDN_OK) return rc;
    for (int32_t sg = 0; sg < n_seg; ++sg) {
        if (seg_ld[sg] < seg_cols[sg + 1] - seg_cols[sg]) return GDN_ERR_SHAPE;
        if (T > 0 && !seg_y[sg]) return GDN_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(seg_y[sg]) & (out_dtype == GDN_BF16 ? 7u : 15u)) || (seg_ld[sg] & 3)) return GDN_ERR_ALIGN;
    }
    if (T == 0) return GDN_OK;
    LinearArgs a = {};
    a.x = x; a.w = w; a.bias = bias; a.y = seg_y[0];
    a.ldx = ldx; a.ldw = ldw; a.ldy = seg_ld[0];
    a.T = T; a.N = N; a.K = K;
    a.n_seg = n_seg;
    for (int32_t sg = 0; sg < n_seg; ++sg) {
        a.seg_col[sg] = seg_cols[sg];
        a.seg_y[sg] = seg_y[sg];
        a.seg_ld[sg] = seg_ld[sg];
    }
    for (int32_t sg = n_seg; sg <= LIN_MAX_SEG; ++sg) a.seg_col[sg] = N;
    return linear_launch(a, out_dtype, (hipStream_t)stream_);
}

extern "C" int32_t gdn_linear_plan(int64_t T, int32_t N, int32_t K, int32_t* shape, int32_t* cols, int32_t* rest_shape) {
    if (T <= 0 || N <= 0 || K <= 0) return GDN_ERR_COUNT;
    if (K % 64 != 0) return GDN_ERR_SHAPE;
    if (!shape || !cols || !rest_shape) return GDN_ERR_NULL;
    const LinearPlan p = plan_linear(T, N, K);
    *shape = p.shape;
    *cols = p.cols;
    *rest_shape = p.rest_shape;
    return GDN_OK;
}

extern "C" int32_t gdn_linear_tune(int32_t shape) {
    return g_linear_shape.exchange(shape < 0 || shape > 5 ? -1 : shape);
}

extern "C" int32_t gdn_linear_act(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, const gdn_linear_epilogue* epi, void* y,
                                  int64_t ldy, int32_t out_dtype, int64_t T, int32_t N, int32_t K, void* stream_) {
    if (!epi) return GDN_ERR_NULL;
    int32_t rc = linear_checks(x, ldx, w, ldw, bias, out_dtype, T, N, K);
    if (rc != GDN_OK) return rc;
    if (epi->act < GDN_ACT_NONE || epi->act > GDN_ACT_SIGMOID || (epi->bias_up && !epi->w_up) || ldy < N) return GDN_ERR_SHAPE;
    if (epi->w_up && epi->ldw_up < K) return GDN_ERR_SHAPE;
    if (epi->residual && (!dtype_known(epi->res_dtype) || epi->ldr < N)) return GDN_ERR_SHAPE;
    if (T == 0 || N == 0) return GDN_OK;
    if (!y) return GDN_ERR_NULL;
    const int es = dtype_bytes(out_dtype), rs = dtype_bytes(epi->res_dtype);
    if (off_align(y, es == 2 ? 8 : 16) || (ldy & 3)) return GDN_ERR_ALIGN;
    if (epi->w_up && (off_align(epi->w_up, 16) || (epi->ldw_up & 7))) return GDN_ERR_ALIGN;
    if (off_align(epi->bias_up, 4)) return GDN_ERR_ALIGN;
    if (epi->residual && (off_align(epi->residual, rs == 2 ? 8 : 16) || (epi->ldr & 3))) return GDN_ERR_ALIGN;
    if (epi->w_up && epi->ldw_up >= ((int64_t)1 << 22)) return GDN_ERR_COUNT;
    // a kernel of a few rows has some 32 threads to an output, a launch less than 2^32, and the tensors' spans have to fit 63 bits
    const int64_t most = std::min((int64_t)1 << 30, ((int64_t)1 << 60) / T);
    if (N >= 1 << 24 || ldy > most || (epi->residual && epi->ldr > most)) return GDN_ERR_COUNT;
    const Rows out(y, T, ldy * es, (int64_t)N * es), res(epi->residual, T, epi->ldr * rs, (int64_t)N * rs);
    if (share_bytes(out, Rows(x, T, ldx * 2, (int64_t)K * 2)) || share_bytes(out, Rows(w, N, ldw * 2, (int64_t)K * 2)) ||
        share_bytes(out, Rows(epi->w_up, N, epi->ldw_up * 2, (int64_t)K * 2)) || share_bytes(out, Rows(bias, 1, (int64_t)N * 4, (int64_t)N * 4)) ||
        share_bytes(out, Rows(epi->bias_up, 1, (int64_t)N * 4, (int64_t)N * 4)) || (share_bytes(out, res) && !same_rows(out, res)))
        return GDN_ERR_SLOT_HAZARD;
    LinearActArgs a = {};
    a.x = x; a.w = w; a.bias = bias; a.y = y;
    a.ldx = ldx; a.ldw = ldw; a.ldy = ldy;
    a.T = T; a.N = N; a.K = K;
    a.w_up = epi->w_up; a.ldw_up = epi->ldw_up; a.bias_up = epi->bias_up;
    a.residual = epi->residual; a.ldr = epi->ldr; a.res_f32 = epi->res_dtype == GDN_F32;
    a.act = epi->act; a.scale = epi->scale;
    hipStream_t stream = (hipStream_t)stream_;
    const bool bf = out_dtype == GDN_BF16;
    const LinearPlan p = plan_act(T, N, K, epi->w_up != nullptr);
    if (p.cols == N) return launch_act_shape(a, p.shape, bf, stream);
    rc = launch_act_shape(act_range(a, 0, p.cols, es), p.shape, bf, stream);
    return rc != GDN_OK ? rc : launch_act_shape(act_range(a, p.cols, N, es), p.rest_shape, bf, stream);
}

extern "C" int32_t gdn_linear_act_plan(int64_t T, int32_t N, int32_t K, int32_t gated, int32_t* shape, int32_t* cols, int32_t* rest_shape) {
    if (T <= 0 || N <= 0 || K <= 0) return GDN_ERR_COUNT;
    if (K % 64 != 0 || gated < 0 || gated > 1) return GDN_ERR_SHAPE;
    if (!shape || !cols || !rest_shape) return GDN_ERR_NULL;
    const LinearPlan p = plan_act(T, N, K, gated != 0);
    *shape = p.shape;
    *cols = p.cols;
    *rest_shape = p.rest_shape;
    return GDN_OK;
}

extern "C" int32_t gdn_linear_act_tune(int32_t shape) {
    return g_act_shape.exchange(shape < 0 || shape > FEW + 5 ? -1 : shape);
}
