// gdn_block_norm: the residual stream between two blocks, with the norms on both sides (see include/gdn_block.h).
//
// s = r + scale g N_post(y), x = N_pre(s): a few flops for every element read or written once, so memory traffic is all that bounds it.
//
// A row is held in registers from its loads to its stores, 8 adjacent elements to a piece (16 bytes of bf16), so that neither the squares of
// what the mean leaves nor the second norm read it again: one piece to a thread and as many waves as the row has pieces for, up to 16
// (rows of up to 8192), then two or four.  A norm costs one barrier, and few instructions: the vector units, 4 clocks to each instruction
// of a wave, are not far behind the memory (with the waves' sums added up by every thread, and divisions, 928 instructions for 8 elements of
// two layer norms kept them busy for three quarters of the time: 1777 rows of 5120 43 us, now 32).
//
// us, and read and written (a plain copy of 2 GiB 4.9 TB/s):
//   8192 rows of 2048, bf16, the norm in front alone                     26   134 MB   5.2 TB/s     (with one behind the block and a gate per channel 28)
//   8192 of 2048, block and stream fp32, a norm on both sides            46.5 235      5.05
//   1777 of 5120 out of wider buffers, two layer norms, a gate, fp32 stream   32   127      3.9
//   4096 of 4096, bf16, both sides                                       23   134      5.75
//   2048 of 10240, block and stream fp32                                 61.5 294      4.8
//   1000 of 32768, bf16                                                  62   262      4.2          (fp32 block and stream 128, 459 MB, 3.6)
//   a single row 2.4, which a call's host time of 7 covers
// Rows of more than 16384 need more than the 128 registers that 16 waves leave each: 16 to 18 of them, 64 with block and stream in fp32, go to memory and
// back (all operands and weights asked for at once: more of them, 89 us for 1000 of 32768).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "gdn_block.h"
#include "gdn_rows.h"

namespace gdn {
namespace block {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

struct BlockArgs {
    const void *y, *gate, *r;
    const float *w_post, *b_post, *w_pre, *b_pre;
    void *s, *x;
    int64_t ldy, ldg, ldr, lds, ldx;
    int64_t T;
    int32_t D;
    int32_t post, pre, gate_kind, gate_act;
    int32_t in_f32, s_f32, x_f32;
    int32_t waves;
    float eps_post, eps_pre, scale, offset, inv_d;
};

// 8 elements as they lie in memory (fp32 or bf16), so that a row's loads are all on their way before the first is unpacked.
template <bool F32>
struct Piece { u32x4 q[F32 ? 2 : 1]; };
template <bool F32>
__device__ __forceinline__ Piece<F32> fetch(const void* p, int64_t at) {
    Piece<F32> v;
    const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const char*>(p) + at * (F32 ? 4 : 2));
    v.q[0] = q[0];
    if constexpr (F32) v.q[1] = q[1];
    return v;
}
template <bool F32>
__device__ __forceinline__ Piece<F32> nothing() {
    Piece<F32> v;
    v.q[0] = u32x4{0, 0, 0, 0};
    if constexpr (F32) v.q[1] = v.q[0];
    return v;
}
template <bool F32>
__device__ __forceinline__ f32x8 unpack(const Piece<F32>& v) {
    f32x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (F32) o[e] = __uint_as_float(v.q[e / 4][e % 4]);
        else o[e] = __uint_as_float(e & 1 ? v.q[0][e / 2] & 0xffff0000u : v.q[0][e / 2] << 16);
    }
    return o;
}
__device__ __forceinline__ void put(void* p, int64_t at, int f32, const f32x8& v) {
    if (f32) {
        f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + at);
        q[0] = f32x4{v[0], v[1], v[2], v[3]};
        q[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        *reinterpret_cast<bf16x8*>(static_cast<uint16_t*>(p) + at) = __builtin_convertvector(v, bf16x8);
    }
}
__device__ __forceinline__ f32x8 fetch_f32(const float* p) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// The sum over a wave, on every lane: moves within the vector unit.
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0x111, 0xf>(v);           // 1, 2, 4, 8 lanes up a row of 16, then the last lane of a row to the next one, and of the first half to the second
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
constexpr int MAX_WAVES = 16;
struct alignas(16) Parts { float sum, mean, squares, count; };

// A norm's weights (with their offset) for a thread's pieces.
template <int PIECES>
struct Weights { f32x8 w[PIECES]; };
template <int PIECES>
__device__ __forceinline__ void fetch_weights(Weights<PIECES>& q, const float* w, float offset, int first, int stride, int D) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * stride;
        q.w[i] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c >= D) continue;
        q.w[i] = fetch_f32(w + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) q.w[i][e] += offset;
    }
}

// v <- N(v) over the row.  Every wave takes the mean of its own elements and the squares of what that leaves; the waves' meet in LDS behind one barrier,
// a wave's to a lane, the squares about the row's mean by  sum (v - m)^2 = sum over waves of (sum (v - m_w)^2 + n_w (m_w - m)^2).  `part`: two sets, between which
// `turn` alternates, so one barrier is enough for each norm.  The same on every thread, and the same whenever it runs.
template <int PIECES>
__device__ __forceinline__ void normalise(f32x8 (&v)[PIECES], int kind, const Weights<PIECES>& kept, const float* w, const float* bias, float eps, const BlockArgs& a, int first, int stride,
                                          Parts (*part)[MAX_WAVES], int& turn, int wave) {
    const int waves = a.waves;
    const bool layer = kind == GDN_NORM_LAYER;
    // the biases: asked for in front of the sums, not behind the barrier, where there are registers for them
    f32x8 early = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (PIECES == 1 && bias && first < a.D) early = fetch_f32(bias + first);
    Parts mine = {0.f, 0.f, 0.f, 0.f};
    if (layer) {
        int n = 0;                                               // the wave's elements
#pragma unroll
        for (int i = 0; i < PIECES; ++i) n += min(max(a.D - i * stride - (waves == 1 ? 0 : wave * 512), 0), 512);
        mine.count = (float)n;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) mine.sum += v[i][e];     // (pieces behind the row's end hold zeros)
        mine.sum = wave_sum(mine.sum);
        mine.mean = mine.sum * (n == 512 ? 1.f / 512.f : __builtin_amdgcn_rcpf(mine.count));
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (first + i * stride < a.D)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v[i][e] - mine.mean;
                mine.squares = fmaf(d, d, mine.squares);
            }
    mine.squares = wave_sum(mine.squares);
    float mean = mine.mean, squares = mine.squares;
    if (waves > 1) {
        const int lane = threadIdx.x & 63;
        Parts* p = part[turn];
        turn ^= 1;
        if (lane == 0) p[wave] = mine;
        __syncthreads();
        Parts other = {0.f, 0.f, 0.f, 0.f};                      // a wave's parts to a lane
        if (lane < waves) other = p[lane];
        if (layer) {
            mean = wave_sum(other.sum) * a.inv_d;
            const float d = other.mean - mean;
            other.squares = fmaf(other.count * d, d, other.squares);
        }
        squares = wave_sum(other.squares);
    }
    const float inv = __builtin_amdgcn_rsqf(fmaf(squares, a.inv_d, eps));
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * stride;
        if (c >= a.D) continue;
        f32x8 b = early;
        if (PIECES > 1 && bias) b = fetch_f32(bias + c);
        f32x8 g;
        if constexpr (PIECES == 1) g = kept.w[0];
        else g = fetch_f32(w + c) + a.offset;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = fmaf((v[i][e] - mean) * inv, g[e], b[e]);
    }
}

// `a.waves` waves to a row, PIECES pieces of 8 elements to a thread; with one wave to a row a workgroup has four rows.  A workgroup goes through
// every grid-th row and keeps the weights (and a gate per channel) in registers: read anew for each row those arrays of fp32 are more than the row
// itself, two of bf16 read and two written, and come out of L2.  (Rows wider than 8192 have more than one piece to a thread, and read them where they are used; with four pieces the stream and
// the gate too are asked for only behind the first norm.)
template <int PIECES, bool IN_F32, bool S_F32>
__global__ void __launch_bounds__(64 * MAX_WAVES) gdn_block_norm_kernel(BlockArgs a) {
    __shared__ Parts part[2][MAX_WAVES];
    constexpr bool KEEP = PIECES == 1, LATE = PIECES == 4;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = a.waves, stride = waves * 512;
    const int rows = waves == 1 ? 4 : 1;                         // rows of a workgroup
    const int first = 8 * (waves == 1 ? tid & 63 : tid);
    int turn = 0;
    Weights<PIECES> post, pre, channel;
    if (KEEP && a.post != GDN_NORM_NONE) fetch_weights(post, a.w_post, a.offset, first, stride, a.D);
    if (KEEP && a.pre != GDN_NORM_NONE) fetch_weights(pre, a.w_pre, a.offset, first, stride, a.D);
    if (KEEP && a.gate_kind == GDN_GATE_CHANNEL) fetch_weights(channel, static_cast<const float*>(a.gate), 0.f, first, stride, a.D);
    // (whole waves leave with one wave to a row; with more the loop's count is the workgroup's)
    for (int64_t t = (int64_t)blockIdx.x * rows + (waves == 1 ? wave : 0); t < a.T; t += (int64_t)gridDim.x * rows) {
        Piece<IN_F32> py[PIECES], pg[PIECES];
        Piece<S_F32> pr[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = first + i * stride;
            py[i] = pg[i] = nothing<IN_F32>();
            pr[i] = nothing<S_F32>();
            if (c >= a.D) continue;
            if (a.y) py[i] = fetch<IN_F32>(a.y, t * a.ldy + c);
            if (LATE) continue;
            if (a.r) pr[i] = fetch<S_F32>(a.r, t * a.ldr + c);
            if (a.gate_kind == GDN_GATE_ELEMENT) pg[i] = fetch<IN_F32>(a.gate, t * a.ldg + c);
        }
        float one_gate = a.scale;
        if (a.gate_kind == GDN_GATE_TOKEN) {
            float g = IN_F32 ? static_cast<const float*>(a.gate)[t * a.ldg] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.gate)[t * a.ldg] << 16);
            if (a.gate_act) g = 1.f / (1.f + expf(-g));
            one_gate *= g;
        }
        f32x8 v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) v[i] = unpack(py[i]);
        if (a.post != GDN_NORM_NONE) normalise(v, a.post, post, a.w_post, a.b_post, a.eps_post, a, first, stride, part, turn, wave);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = first + i * stride;
            if (c >= a.D) continue;
            if (LATE && a.r) pr[i] = fetch<S_F32>(a.r, t * a.ldr + c);
            if (LATE && a.gate_kind == GDN_GATE_ELEMENT) pg[i] = fetch<IN_F32>(a.gate, t * a.ldg + c);
            if (a.gate_kind == GDN_GATE_ELEMENT || a.gate_kind == GDN_GATE_CHANNEL) {
                f32x8 g = unpack(pg[i]);
                if (a.gate_kind == GDN_GATE_CHANNEL) g = KEEP ? channel.w[i] : fetch_f32(static_cast<const float*>(a.gate) + c);
                if (a.gate_act)
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[e] = __builtin_amdgcn_rcpf(1.f + __expf(-g[e]));
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] *= g[e];
            }
            const f32x8 r = unpack(pr[i]);
            if (a.y)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = a.r ? fmaf(one_gate, v[i][e], r[e]) : one_gate * v[i][e];
            else v[i] = r;
            if (a.s) put(a.s, t * a.lds + c, S_F32, v[i]);
        }
        if (a.pre == GDN_NORM_NONE) continue;
        normalise(v, a.pre, pre, a.w_pre, a.b_pre, a.eps_pre, a, first, stride, part, turn, wave);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = first + i * stride;
            if (c < a.D) put(a.x, t * a.ldx + c, a.x_f32, v[i]);
        }
    }
}

template <int PIECES, bool IN_F32, bool S_F32>
void launch_kernel(const BlockArgs& a, unsigned blocks, unsigned threads, hipStream_t stream) {
    hipLaunchKernelGGL((gdn_block_norm_kernel<PIECES, IN_F32, S_F32>), dim3(blocks), dim3(threads), 0, stream, a);
}
template <int PIECES>
hipError_t launch(BlockArgs a, hipStream_t stream) {
    a.waves = (a.D + 512 * PIECES - 1) / (512 * PIECES);
    // As many workgroups as are on the chip at once, at 24 waves to a compute unit, which is what the registers of the kernels of rows up to 8192 leave (4096 rows of 8192, 16 waves
    // each, 58 us in 256 workgroups, 82 in 320).  With block and stream in fp32 it is 20, and 16 for wider rows, so that some widths (fp32: up to 2048, 2561 to 4096, 5121 to 6144; any type:
    // 8193 to 12288, 16385 to 24576) get more workgroups than fit: 8192 rows of 2048 and 4096 of 4096 in fp32 run at 5.05 TB/s all the same, 2048 of 10240 at 4.8.
    const int per_block = a.waves == 1 ? 4 : a.waves;            // waves
    const unsigned blocks = (unsigned)std::min<int64_t>(a.waves == 1 ? (a.T + 3) / 4 : a.T, (int64_t)chip_cus() * (24 / per_block)), threads = 64u * per_block;
    if (a.in_f32) a.s_f32 ? launch_kernel<PIECES, true, true>(a, blocks, threads, stream) : launch_kernel<PIECES, true, false>(a, blocks, threads, stream);
    else a.s_f32 ? launch_kernel<PIECES, false, true>(a, blocks, threads, stream) : launch_kernel<PIECES, false, false>(a, blocks, threads, stream);
    return hipGetLastError();
}

int32_t check(const gdn_block_shape* p, const void* y, int64_t ldy, const void* gate, int64_t ldg, const float* w_post, const float* b_post,
              const void* r, int64_t ldr, const float* w_pre, const float* b_pre, void* s, int64_t lds, void* x, int64_t ldx, int64_t T) {
    if (!p) return GDN_ERR_NULL;
    if (T < 0) return GDN_ERR_COUNT;
    if (p->D < 8 || p->D > 32768 || !dtype_known(p->in_dtype) || !dtype_known(p->s_dtype) || !dtype_known(p->x_dtype)) return GDN_ERR_SHAPE;
    if (p->post < 0 || p->post > GDN_NORM_LAYER || p->pre < 0 || p->pre > GDN_NORM_LAYER || p->gate < 0 || p->gate > GDN_GATE_CHANNEL ||
        p->gate_act < 0 || p->gate_act > 1)
        return GDN_ERR_SHAPE;
    if (!(p->eps_post >= 0.f) || !(p->eps_pre >= 0.f) || !std::isfinite(p->eps_post) || !std::isfinite(p->eps_pre)) return GDN_ERR_SHAPE;
    if (p->D & 7) return GDN_ERR_ALIGN;
    if (T == 0) return GDN_OK;
    const int64_t D = p->D;
    if (!y && !r) return GDN_ERR_NULL;
    if (!y && (p->post != GDN_NORM_NONE || p->gate != GDN_GATE_NONE)) return GDN_ERR_SHAPE;
    if (p->pre == GDN_NORM_NONE ? (x || !s) : !x) return x ? GDN_ERR_SHAPE : GDN_ERR_NULL;
    if ((p->post != GDN_NORM_NONE && !w_post) || (p->pre != GDN_NORM_NONE && !w_pre) || (p->gate != GDN_GATE_NONE && !gate)) return GDN_ERR_NULL;
    struct { const void* at; int64_t ld; } rows[4] = {{y, ldy}, {r, ldr}, {s, lds}, {x, ldx}};
    for (const auto& q : rows) {
        if (!q.at) continue;
        if (q.ld < D) return GDN_ERR_SHAPE;
        if (off_align(q.at, 16) || (q.ld & 7)) return GDN_ERR_ALIGN;
    }
    const int in = dtype_bytes(p->in_dtype), sb = dtype_bytes(p->s_dtype), xb = dtype_bytes(p->x_dtype);
    if (p->gate == GDN_GATE_ELEMENT) {
        if (ldg < D) return GDN_ERR_SHAPE;
        if (off_align(gate, 16) || (ldg & 7)) return GDN_ERR_ALIGN;
    } else if (p->gate == GDN_GATE_TOKEN) {
        if (ldg < 1) return GDN_ERR_SHAPE;
        if (off_align(gate, in)) return GDN_ERR_ALIGN;
    } else if (p->gate == GDN_GATE_CHANNEL && off_align(gate, 16)) {
        return GDN_ERR_ALIGN;
    }
    for (const float* q : {p->post != GDN_NORM_NONE ? w_post : nullptr, p->post != GDN_NORM_NONE ? b_post : nullptr,
                           p->pre != GDN_NORM_NONE ? w_pre : nullptr, p->pre != GDN_NORM_NONE ? b_pre : nullptr})
        if (off_align(q, 16)) return GDN_ERR_ALIGN;
    // the tensors' spans have to fit 63 bits, and a workgroup's number 31
    int64_t most = std::max(std::max(y ? ldy : 0, r ? ldr : 0), std::max(s ? lds : 0, x ? ldx : 0));
    if (p->gate == GDN_GATE_ELEMENT || p->gate == GDN_GATE_TOKEN) most = std::max(most, ldg);
    if (T > INT32_MAX || most > std::min((int64_t)1 << 40, ((int64_t)1 << 60) / T)) return GDN_ERR_COUNT;

    const Rows outs[2] = {Rows(s, T, lds * sb, D * sb), Rows(x, T, ldx * xb, D * xb)};
    if (share_bytes(outs[0], outs[1])) return GDN_ERR_SLOT_HAZARD;
    const Rows ins[3] = {Rows(y, T, ldy * in, D * in), Rows(r, T, ldr * sb, D * sb),
                         Rows(p->gate == GDN_GATE_ELEMENT ? gate : nullptr, T, ldg * in, D * in)};
    const Rows fixed[6] = {Rows(p->gate == GDN_GATE_TOKEN ? gate : nullptr, T, ldg * in, in), Rows(p->gate == GDN_GATE_CHANNEL ? gate : nullptr, 1, D * 4, D * 4),
                           Rows(p->post != GDN_NORM_NONE ? w_post : nullptr, 1, D * 4, D * 4), Rows(p->post != GDN_NORM_NONE ? b_post : nullptr, 1, D * 4, D * 4),
                           Rows(p->pre != GDN_NORM_NONE ? w_pre : nullptr, 1, D * 4, D * 4), Rows(p->pre != GDN_NORM_NONE ? b_pre : nullptr, 1, D * 4, D * 4)};
    for (const Rows& o : outs) {
        for (const Rows& i : ins)
            if (share_bytes(o, i) && !same_rows(o, i)) return GDN_ERR_SLOT_HAZARD;
        for (const Rows& i : fixed)
            if (share_bytes(o, i)) return GDN_ERR_SLOT_HAZARD;
    }
    return GDN_OK;
}

}  // namespace block
}  // namespace gdn

using namespace gdn;
using namespace gdn::block;

extern "C" int32_t gdn_block_norm(const gdn_block_shape* p, const void* y, int64_t ldy, const void* gate, int64_t ldg, const float* w_post,
                                  const float* b_post, const void* r, int64_t ldr, const float* w_pre, const float* b_pre, void* s, int64_t lds,
                                  void* x, int64_t ldx, int64_t T, void* stream_) {
    const int32_t rc = check(p, y, ldy, gate, ldg, w_post, b_post, r, ldr, w_pre, b_pre, s, lds, x, ldx, T);
    if (rc != GDN_OK || T == 0) return rc;
    BlockArgs a = {};
    a.y = y; a.gate = gate; a.r = r; a.s = s; a.x = x;
    a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre; a.b_pre = b_pre;
    a.ldy = ldy; a.ldg = ldg; a.ldr = ldr; a.lds = lds; a.ldx = ldx;
    a.T = T; a.D = p->D;
    a.post = p->post; a.pre = p->pre; a.gate_kind = p->gate; a.gate_act = p->gate_act;
    a.in_f32 = p->in_dtype == GDN_F32; a.s_f32 = p->s_dtype == GDN_F32; a.x_f32 = p->x_dtype == GDN_F32;
    a.eps_post = p->eps_post; a.eps_pre = p->eps_pre; a.scale = p->scale; a.offset = p->offset;
    a.inv_d = 1.f / (float)p->D;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    const hipError_t e = p->D <= 8192 ? launch<1>(a, stream) : p->D <= 16384 ? launch<2>(a, stream) : launch<4>(a, stream);
    return e == hipSuccess ? GDN_OK : GDN_ERR_HIP - (int32_t)e;
}
