// gdn_block_norm: the residual stream between two blocks, with the norms on both sides (see include/gdn_block.h).
//
// s = r + scale g N_post(y), x = N_pre(s): a few flops for every element read or written once, so memory traffic is all that
// bounds it.  A row is held in registers from its loads to its stores, 8 adjacent elements to a piece (16 bytes of bf16), up
// to four pieces a thread, so that neither the squares of what the mean leaves nor the second norm read it again.  A row is
// dealt to 1, 4 or 16 waves: the fewest that hold it where there are rows enough to fill the chip (a wave by itself needs no
// barrier for its sums), more where there are few and a row's own latency is the time.
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
    float eps_post, eps_pre, scale, offset, inv_d;
};

// 8 elements as they lie in memory, so that a row's loads are all on their way before the first is unpacked.
struct Piece { u32x4 lo, hi; };
__device__ __forceinline__ Piece fetch(const void* p, int64_t at, int f32) {
    Piece v = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (f32) {
        const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + at);
        v.lo = q[0];
        v.hi = q[1];
    } else {
        v.lo = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
    }
    return v;
}
__device__ __forceinline__ f32x8 unpack(const Piece& v, int f32) {
    f32x8 o;
    if (f32) {
        const f32x4 a = __builtin_bit_cast(f32x4, v.lo), b = __builtin_bit_cast(f32x4, v.hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { o[i] = a[i]; o[i + 4] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = __uint_as_float(v.lo[i] << 16);
            o[2 * i + 1] = __uint_as_float(v.lo[i] & 0xffff0000u);
        }
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

// The sum over a row's waves, the same on every thread and the same whenever it runs: a butterfly over the lanes, then the waves' sums in order.
// `part`: WAVES floats of this row; `turn` alternates between two sets, so one barrier is enough for each sum.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float (*part)[WAVES], int& turn, int wave) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    if (WAVES == 1) return v;
    float* p = part[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) p[wave] = v;
    __syncthreads();
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) total += p[i];
    return total;
}

// v <- N(v) over the row; w, b: the row's parameters (b may be null).
template <int WAVES, int PIECES>
__device__ __forceinline__ void normalise(f32x8 (&v)[PIECES], int kind, const float* w, const float* b, float offset, float eps, float inv_d, int D,
                                          int first, float (*part)[WAVES], int& turn, int wave) {
    if (kind == GDN_NORM_LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[i][e];          // (pieces behind the row's end hold zeros)
        const float mean = row_sum<WAVES>(sum, part, turn, wave) * inv_d;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (first + i * WAVES * 512 < D)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] -= mean;
    }
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = fmaf(v[i][e], v[i][e], squares);
    const float inv = 1.f / sqrtf(row_sum<WAVES>(squares, part, turn, wave) * inv_d + eps);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * WAVES * 512;
        if (c >= D) continue;
        const f32x8 wv = fetch_f32(w + c);
        f32x8 bv = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (b) bv = fetch_f32(b + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e] * inv, wv[e] + offset, bv[e]);
    }
}

// WAVES waves to a row, PIECES pieces of 8 elements to a thread; a workgroup of at least four waves.
template <int WAVES, int PIECES>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) gdn_block_norm_kernel(BlockArgs a) {
    __shared__ float part[2][WAVES];
    constexpr int ROWS = WAVES == 1 ? 4 : 1;                     // rows of a workgroup
    const int tid = threadIdx.x, wave = tid >> 6;
    const int64_t t = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? wave : 0);
    if (t >= a.T) return;                                        // (whole waves; with more waves to a row the grid is the rows)
    const int first = 8 * (WAVES == 1 ? tid & 63 : tid);
    int turn = 0;
    Piece py[PIECES], pr[PIECES], pg[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * WAVES * 512;
        py[i] = pr[i] = pg[i] = Piece{{0, 0, 0, 0}, {0, 0, 0, 0}};
        if (c >= a.D) continue;
        if (a.y) py[i] = fetch(a.y, t * a.ldy + c, a.in_f32);
        if (a.r) pr[i] = fetch(a.r, t * a.ldr + c, a.s_f32);
        if (a.gate_kind == GDN_GATE_ELEMENT) pg[i] = fetch(a.gate, t * a.ldg + c, a.in_f32);
    }
    float one_gate = a.scale;
    if (a.gate_kind == GDN_GATE_TOKEN) {
        float g = a.in_f32 ? static_cast<const float*>(a.gate)[t * a.ldg]
                           : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.gate)[t * a.ldg] << 16);
        if (a.gate_act) g = 1.f / (1.f + expf(-g));
        one_gate *= g;
    }
    f32x8 v[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) v[i] = unpack(py[i], a.in_f32);
    if (a.post != GDN_NORM_NONE)
        normalise<WAVES, PIECES>(v, a.post, a.w_post, a.b_post, a.offset, a.eps_post, a.inv_d, a.D, first, part, turn, wave);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * WAVES * 512;
        if (c >= a.D) continue;
        if (a.gate_kind == GDN_GATE_ELEMENT || a.gate_kind == GDN_GATE_CHANNEL) {
            f32x8 g = a.gate_kind == GDN_GATE_ELEMENT ? unpack(pg[i], a.in_f32) : fetch_f32(static_cast<const float*>(a.gate) + c);
            if (a.gate_act)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = 1.f / (1.f + __expf(-g[e]));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= g[e];
        }
        const f32x8 r = unpack(pr[i], a.s_f32);
        if (a.y)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = a.r ? fmaf(one_gate, v[i][e], r[e]) : one_gate * v[i][e];
        else v[i] = r;
        if (a.s) put(a.s, t * a.lds + c, a.s_f32, v[i]);
    }
    if (a.pre == GDN_NORM_NONE) return;
    normalise<WAVES, PIECES>(v, a.pre, a.w_pre, a.b_pre, a.offset, a.eps_pre, a.inv_d, a.D, first, part, turn, wave);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int c = first + i * WAVES * 512;
        if (c < a.D) put(a.x, t * a.ldx + c, a.x_f32, v[i]);
    }
}

template <int WAVES, int PIECES>
hipError_t launch(const BlockArgs& a, hipStream_t stream) {
    const int64_t blocks = WAVES == 1 ? (a.T + 3) / 4 : a.T;
    hipLaunchKernelGGL((gdn_block_norm_kernel<WAVES, PIECES>), dim3((unsigned)blocks), dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, stream, a);
    return hipGetLastError();
}

template <int WAVES>
hipError_t launch_pieces(const BlockArgs& a, int pieces, hipStream_t stream) {
    return pieces <= 1 ? launch<WAVES, 1>(a, stream) : pieces <= 2 ? launch<WAVES, 2>(a, stream) : launch<WAVES, 4>(a, stream);
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
    // every byte offset of a row has to fit 63 bits, and a workgroup's number 31
    int64_t most = std::max(std::max(y ? ldy : 0, r ? ldr : 0), std::max(s ? lds : 0, x ? ldx : 0));
    if (p->gate == GDN_GATE_ELEMENT || p->gate == GDN_GATE_TOKEN) most = std::max(most, ldg);
    if (T > INT32_MAX || most > ((int64_t)1 << 40)) return GDN_ERR_COUNT;

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
    const int pieces = (p->D / 8 + 63) / 64;                     // of a wave that has the row by itself
    hipError_t e;
    if (pieces > 16) e = launch_pieces<16>(a, (pieces + 15) / 16, stream);
    else if (pieces > 4 || (pieces > 1 && T < 4096)) e = launch_pieces<4>(a, (pieces + 3) / 4, stream);
    else e = launch_pieces<1>(a, pieces, stream);
    return e == hipSuccess ? GDN_OK : GDN_ERR_HIP - (int32_t)e;
}
