// gdn_moe: host side of a mixture of experts (see include/gdn_moe.h, kernels in gdn_moe_kernel.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "gdn_moe.h"
#include "gdn_moe_kernel.h"
#include "gdn_rows.h"

namespace gdn {
namespace moe {

inline int32_t hip_err(hipError_t e) { return e == hipSuccess ? GDN_OK : GDN_ERR_HIP - (int32_t)e; }

int32_t check_shape(const gdn_moe_shape* s, int64_t T) {
    if (!s) return GDN_ERR_NULL;
    if (T < 0) return GDN_ERR_COUNT;
    if (s->E < 1 || s->E > MAX_E || s->k < 1 || s->k > MAX_K || s->k > s->E) return GDN_ERR_SHAPE;
    if (s->D < 64 || s->D > 32768 || s->D % 64 || s->F < 64 || s->F > 32768 || s->F % 64) return GDN_ERR_SHAPE;
    if (s->act < GDN_ACT_NONE || s->act > GDN_ACT_SIGMOID || s->score < 0 || s->score > GDN_SCORE_SIGMOID || s->normalise < 0 || s->normalise > 1 ||
        !dtype_known(s->router_dtype) || !std::isfinite(s->routed_scale))
        return GDN_ERR_SHAPE;
    if (T >= ((int64_t)1 << 24) || T * s->k >= ((int64_t)1 << 24)) return GDN_ERR_COUNT;
    return GDN_OK;
}

// Byte offsets of the workspace's arrays.
struct Layout { int64_t logits, ids, weights, counts, list, table, h, part, end; };
int64_t most_tiles(const gdn_moe_shape& s, int64_t T) {         // of 64 rows, the smallest: every expert may have one that is not full
    return T * s.k / 64 + std::min<int64_t>(s.E, T * s.k);
}
Layout layout(const gdn_moe_shape& s, int64_t T) {
    Layout w;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    w.logits = take(T * s.E * 4);
    w.ids = take(T * s.k * 4);
    w.weights = take(T * s.k * 4);
    w.counts = take(s.E * 4);
    w.list = take(T * s.E * 4);
    w.table = take((most_tiles(s, T) + 1) * (int64_t)sizeof(linear::ExpertTile));
    w.h = take(T * s.k * s.F * 2);
    w.part = take(T * s.k * s.D * 4);
    w.end = at;
    return w;
}

template <int TT, int TE, int U>
void launch_logits(const MoeArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((moe_logits_few_kernel<TT, TE, U>), dim3((unsigned)((a.E + 4 * TE - 1) / (4 * TE)), (unsigned)((a.T + TT - 1) / TT)), dim3(256), 0, stream, a);
}
template <void (*KERNEL)(MoeArgs)>
hipError_t launch_few_kernel(dim3 grid, int waves, int smem, const MoeArgs& a, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(KERNEL), smem, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(KERNEL, grid, dim3(64 * waves), smem, stream, a);
    return hipGetLastError();
}
template <typename C, int P>
hipError_t launch_up_few(const MoeArgs& a, hipStream_t stream) {
    return launch_few_kernel<moe_up_few_kernel<C, P>>(dim3((unsigned)(2 * a.F / C::WR), (unsigned)(a.T * a.k)), C::WAVES, C::SMEM, a, stream);
}
template <typename C>
hipError_t launch_down_few(const MoeArgs& a, hipStream_t stream) {
    return launch_few_kernel<moe_down_few_kernel<C>>(dim3((unsigned)(a.D / C::WR), (unsigned)a.T), C::WAVES, C::SMEM, a, stream);
}
// f(a constant of how many experts a lane looks at)
template <typename F>
auto by_experts(int E, F f) {
    const int per_lane = (E + 63) / 64;
    return per_lane <= 1   ? f(std::integral_constant<int, 1>())
           : per_lane <= 2 ? f(std::integral_constant<int, 2>())
           : per_lane <= 4 ? f(std::integral_constant<int, 4>())
           : per_lane <= 8 ? f(std::integral_constant<int, 8>())
                           : f(std::integral_constant<int, 16>());
}
void launch_choices(const MoeArgs& a, hipStream_t stream) {
    by_experts(a.E, [&](auto p) { hipLaunchKernelGGL((moe_route_kernel<decltype(p)::value>), dim3((unsigned)((a.T + 3) / 4)), dim3(256), 0, stream, a); });
}
hipError_t launch_few(const MoeArgs& a, hipStream_t stream) {
    // Where all workgroups of the first product are on the chip at once, each of them chooses anew: a launch less.  In more rounds the choice, 2 us and
    // with many experts 4, would come once in each.
    //   us, chosen inside / by a launch:  128 experts, k 8, F 768: 1 token 25.2 / 27.0, 2 35 / 35;  512 experts, F 256: 4 20.8 / 22.6, 8 29.7 / 27.3, 32 93 / 65;
    //                                     512, k 10, F 512: 16 209 / 172
    // Workgroups of 16 of F, two to a compute unit, or of 8, three: the smaller spread more evenly until there are many, or until they are more than a round.
    //   us, of 16 / of 8, by the workgroups of 16 that there are:  128 experts, k 8, D 2048, F 768: 384 23.8 / 22.8, 768 35.3 / 33.1, 1536 57 / 55, twice that 98 / 101;
    //                                     256, F 512: 512 25.4 / 28.4;  64, k 6, F 1408: 528 30.9 / 29.8, 2112 73 / 75
    const int64_t wide_ones = (int64_t)a.T * a.k * (a.F / 16), cus = chip_cus();
    const bool inside = wide_ones <= 2 * cus, wide = inside ? 2 * wide_ones > 3 * cus : wide_ones > 6 * cus;
    hipError_t e;
    if (inside) {
        e = by_experts(a.E, [&](auto p) { return wide ? launch_up_few<few::Few<1, 32, 4, 3>, decltype(p)::value>(a, stream) : launch_up_few<few::Few<1, 16, 4, 3>, decltype(p)::value>(a, stream); });
    } else {
        launch_choices(a, stream);
        e = wide ? launch_up_few<few::Few<1, 32, 4, 3>, 0>(a, stream) : launch_up_few<few::Few<1, 16, 4, 3>, 0>(a, stream);
    }
    if (e != hipSuccess) return e;
    // a narrow output in workgroups of 8 of its rows, so that there is one for every compute unit
    return a.T * (a.D / 16) < chip_cus() ? launch_down_few<few::Few<1, 8, 4, 6>>(a, stream) : launch_down_few<few::Few<1, 16, 4, 4>>(a, stream);
}

void launch_route(const MoeArgs& a, hipStream_t stream) {
    // In one workgroup while its compute unit has no more to choose than that (16 tokens of 128 experts 23.0 us a call, 20 so 24.2 and in two launches 23.9; of 512 34.9, in two some 31; and 16 keys
    // a lane do not fit the registers of 16 waves).
    if (a.T <= FEW_TOKENS && a.E <= 512 && a.T * a.E <= 4096) {
        by_experts(a.E, [&](auto p) {
            if constexpr (decltype(p)::value <= 8) hipLaunchKernelGGL((moe_route_few_kernel<decltype(p)::value>), dim3(1), dim3(MAX_E), 0, stream, a);
        });
        return;
    }
    launch_choices(a, stream);
    if ((int64_t)a.T * a.k <= FEW_PAIRS) {
        hipLaunchKernelGGL(moe_lists_few_kernel, dim3(1), dim3(MAX_E), 0, stream, a);
        return;
    }
    hipLaunchKernelGGL(moe_lists_kernel, dim3((unsigned)a.E), dim3(64 * LIST_WAVES), 0, stream, a);
    hipLaunchKernelGGL(moe_table_kernel, dim3(1), dim3(MAX_E), 0, stream, a);
}

// The experts' products, in the projections' tiles.
hipError_t launch_products(const MoeArgs& a, int shape, hipStream_t stream) {
    const int64_t pairs = (int64_t)a.T * a.k;
    linear::ExpertProduct p = {};
    p.list = a.list; p.list_stride = a.T; p.table = a.table; p.n_tiles = a.n_tiles;
    p.most_tiles = (int32_t)(pairs / a.tile_rows + std::min<int64_t>(a.E, pairs));
    p.x = a.x; p.ldx = a.ldx; p.x_rows = a.T; p.div = a.k;
    p.w = a.w_gate_up; p.gated = true; p.act = a.act; p.weights = a.weights;
    p.y = a.h; p.N = a.F; p.K = a.D;
    hipError_t e = linear::launch_expert_product(p, shape, stream);
    if (e != hipSuccess) return e;
    p.x = a.h; p.ldx = a.F; p.x_rows = (int32_t)pairs; p.div = 1;
    p.w = a.w_down; p.gated = false; p.act = GDN_ACT_NONE; p.weights = nullptr;
    p.y = a.part; p.N = a.D; p.K = a.F;
    return linear::launch_expert_product(p, shape, stream);
}

constexpr int FEW = 6, MOST_FEW = 32;
// The kernels of few tokens save launches, some 10 us, and read an expert once for every token that chooses it, out of the caches after the first (20 MB a us).
//   us, theirs / tiles, by tokens:  128 experts, k 8, D 2048, F 768: 1 25 / 33, 4 58 / 67, 8 102 / 108, 16 187 / 165
//                                   8, 2, 2048, 2048: 2 26 / 32, 4 42 / 49, 8 66 / 57
//                                   512, 10, 2048, 512: 8 98 / 115, 16 172 / 188, 32 314 / 291;  1024, 8, 1024, 256: 16 54 / 64, 32 91 / 100
bool few_pays(const gdn_moe_shape& s, int64_t T) {
    const double choices = (double)T * s.k, distinct = s.E * (1.0 - std::pow(1.0 - (double)s.k / s.E, (double)T));
    return (choices - distinct) * 6.0 * s.D * s.F <= 10.0 * 20e6;
}

std::atomic<int32_t> g_moe_shape{-1};
// The tile: by the rounds of tiles over the chip that the two products would take, if the choice is even.  Larger tiles read the weights for fewer row tiles each; of smaller
// ones there are more, which few experts or narrow ones need to occupy the chip, and less of them is empty.
//   us, tiles of 64 x 64 / 128 x 128 / 256 x 256:  64 experts, k 6, D 2048, F 1408: 512 tokens (48 rows an expert) 271 / 274 / 331, 1024 365 / 301 / 353, 1536 477 / 420 / 380, 8192 1826 / 1231 / 1099
//                                                  128, 8, 2048, 768: 2048 526 / 453 / 474;  8, 5, 2112, 256: 363 43 / 59 / 93;  8, 8, 768, 576: 791 65 / 59 / 78
// Over 142 calls (4 to 512 experts, D 256 to 4096, F 128 to 2048, 33 to 8192 tokens) the tiles that are chosen are 0.6 % from the best of the three on average, 13 % at most; chosen
// by the rows alone up to 140 %.
//
// The row tiles that an expert's rows give: their number is near normal, of a variance of its mean, and has a tile more for every whole tile that it passes.
double row_tiles(double rows, int tile) {
    const double s = std::sqrt(rows);
    double n = std::max(0.0, std::floor((rows - 4.0 * s) / tile));           // passed for certain
    for (double j = n; rows - j * tile > -4.0 * s; j += 1.0) n += j == 0.0 ? 1.0 - std::exp(-rows) : 0.5 * std::erfc((j * tile - rows) / (s * 1.4142135623730951));
    return n;
}
int choose_shape(const gdn_moe_shape& s, int64_t T) {
    const double rows = (double)T * s.k / s.E;
    int best = 0;
    double least = 0.0;
    for (const int shape : {0, 3, 2}) {
        const int64_t tiles = (int64_t)std::ceil(s.E * row_tiles(rows, linear::expert_tile_rows(shape)));
        const double t = linear::expert_product_us(shape, tiles, 2 * (int64_t)s.F, s.D) + linear::expert_product_us(shape, tiles, s.D, s.F);
        if (shape == 0 || t < least) { least = t; best = shape; }
    }
    return best;
}

}  // namespace moe
}  // namespace gdn

using namespace gdn;
using namespace gdn::moe;

extern "C" int64_t gdn_moe_workspace_bytes(const gdn_moe_shape* shape, int64_t T) {
    const int32_t rc = check_shape(shape, T);
    return rc != GDN_OK ? rc : layout(*shape, T).end;
}

extern "C" int32_t gdn_moe(const gdn_moe_shape* s, const void* x, int64_t ldx, const void* w_router, const float* choice_bias, const void* w_gate_up,
                           const void* w_down, const void* add, int64_t ld_add, void* y, int64_t ldy, int32_t* ids, float* weights, int64_t T,
                           void* workspace, int64_t workspace_bytes, void* stream_) {
    const int32_t rc = check_shape(s, T);
    if (rc != GDN_OK || T == 0) return rc;
    if (!x || !w_router || !w_gate_up || !w_down || !y) return GDN_ERR_NULL;
    const int64_t D = s->D, F = s->F, E = s->E, most = (int64_t)1 << 30;
    if (ldx < D || ldy < D || (add && ld_add < D)) return GDN_ERR_SHAPE;
    for (const void* p : {x, w_router, w_gate_up, w_down, add, (const void*)y})
        if (off_align(p, 16)) return GDN_ERR_ALIGN;
    if (off_align(choice_bias, 4) || off_align(ids, 4) || off_align(weights, 4)) return GDN_ERR_ALIGN;
    if ((ldx & 7) || (ldy & 7) || (add && (ld_add & 7))) return GDN_ERR_ALIGN;
    if (ldx > most || ldy > most || (add && ld_add > most)) return GDN_ERR_COUNT;
    if ((T - 1) * ldx * 2 + D * 2 > INT32_MAX || T * s->k * F * 2 > INT32_MAX) return GDN_ERR_COUNT;      // the tiles' offsets of rows are 31 bits
    const Layout w = layout(*s, T);
    if (!workspace || off_align(workspace, 16) || workspace_bytes < w.end) return GDN_ERR_WORKSPACE;

    const Rows outs[4] = {Rows(y, T, ldy * 2, D * 2), Rows(ids, 1, T * s->k * 4, T * s->k * 4), Rows(weights, 1, T * s->k * 4, T * s->k * 4),
                          Rows(workspace, 1, w.end, w.end)};
    const int64_t rb = dtype_bytes(s->router_dtype);
    const Rows ins[6] = {Rows(x, T, ldx * 2, D * 2), Rows(w_router, 1, E * D * rb, E * D * rb), Rows(choice_bias, 1, E * 4, E * 4),
                         Rows(w_gate_up, 1, E * 2 * F * D * 2, E * 2 * F * D * 2), Rows(w_down, 1, E * D * F * 2, E * D * F * 2), Rows(add, T, ld_add * 2, D * 2)};
    for (int i = 0; i < 4; ++i) {
        for (int j = i + 1; j < 4; ++j)
            if (share_bytes(outs[i], outs[j])) return GDN_ERR_SLOT_HAZARD;
        for (int j = 0; j < 6; ++j)
            if (share_bytes(outs[i], ins[j]) && !(i == 0 && j == 5 && same_rows(outs[i], ins[j]))) return GDN_ERR_SLOT_HAZARD;
    }

    MoeArgs a = {};
    a.x = static_cast<const uint16_t*>(x); a.w_router = w_router; a.choice_bias = choice_bias;
    a.w_gate_up = static_cast<const uint16_t*>(w_gate_up); a.w_down = static_cast<const uint16_t*>(w_down); a.add = static_cast<const uint16_t*>(add);
    a.y = static_cast<uint16_t*>(y); a.out_ids = ids; a.out_weights = weights;
    a.ldx = ldx; a.ld_add = ld_add; a.ldy = ldy;
    a.T = (int32_t)T; a.E = s->E; a.k = s->k; a.D = s->D; a.F = s->F;
    a.act = s->act; a.score = s->score; a.normalise = s->normalise; a.router_f32 = s->router_dtype == GDN_F32; a.routed_scale = s->routed_scale;
    char* const ws = static_cast<char*>(workspace);
    a.logits = reinterpret_cast<float*>(ws + w.logits); a.ids = reinterpret_cast<int32_t*>(ws + w.ids); a.weights = reinterpret_cast<float*>(ws + w.weights);
    a.counts = reinterpret_cast<int32_t*>(ws + w.counts); a.list = reinterpret_cast<int32_t*>(ws + w.list);
    a.table = reinterpret_cast<linear::ExpertTile*>(ws + w.table) + 1;
    a.n_tiles = reinterpret_cast<int32_t*>(ws + w.table);
    a.h = reinterpret_cast<uint16_t*>(ws + w.h); a.part = reinterpret_cast<float*>(ws + w.part);
    hipStream_t stream = static_cast<hipStream_t>(stream_);

    const int forced = g_moe_shape.load();
    const int shape = forced >= 0 && forced != FEW ? forced : choose_shape(*s, T);
    a.tile_rows = linear::expert_tile_rows(shape);
    if (T * E <= 4096) launch_logits<1, 1, 4>(a, stream);
    else if (T * E <= 8192) launch_logits<2, 1, 4>(a, stream);
    else if (T * E <= 16384) launch_logits<2, 2, 2>(a, stream);
    else hipLaunchKernelGGL(moe_logits_kernel<8>, dim3((unsigned)((T + 15) / 16), (unsigned)((E + 15) / 16)), dim3(64 * 8), 0, stream, a);
    if (forced == FEW ? T <= MOST_FEW : forced < 0 && T <= MOST_FEW && few_pays(*s, T)) return hip_err(launch_few(a, stream));
    launch_route(a, stream);
    const hipError_t e = launch_products(a, shape, stream);
    if (e != hipSuccess) return hip_err(e);
    hipLaunchKernelGGL(moe_sum_kernel, dim3((unsigned)((T * (D / 8) + 255) / 256)), dim3(256), 0, stream, a);
    return hip_err(hipGetLastError());
}

extern "C" int32_t gdn_moe_tune(int32_t shape) {
    return g_moe_shape.exchange(shape == 0 || shape == 2 || shape == 3 || shape == FEW ? shape : -1);
}
