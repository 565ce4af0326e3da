// attn_paged: host side of the paged key/value cache (see include/attn_paged.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <new>
#include <stdexcept>
#include <thread>
#include <vector>

#include "attn_launch.h"
#include "attn_paged.h"
#include "attn_paged_kernel.h"

namespace attn {
namespace {

// Rows are numbered with 32 bits in the kernels, which look up to 64 tiles ahead.
constexpr int64_t MAX_ROWS = INT32_MAX - 8192;

int32_t check_pages(const attn_shape* s, const attn_pages* p) {
    if (!p) return GDN_ERR_NULL;
    if (p->n_pages < 0) return GDN_ERR_COUNT;
    if (p->page_rows < 16 || p->page_rows > 256 || (p->page_rows & (p->page_rows - 1)) != 0) return GDN_ERR_SHAPE;
    if (p->page_stride < 0 || p->page_stride % 8 != 0) return GDN_ERR_ALIGN;
    const int64_t elems = (int64_t)s->H_kv * p->page_rows * s->d;
    if (elems * 2 > INT32_MAX || p->page_stride < elems) return GDN_ERR_SHAPE;
    return GDN_OK;
}

inline int shift_of(const attn_pages* p) { return __builtin_ctz((unsigned)p->page_rows); }

// The new tokens of every request.
int32_t check_lengths(int32_t n_req, const int32_t* cu, const int32_t* start, std::vector<int32_t>& len) {
    if (!cu || !start) return GDN_ERR_NULL;
    if (cu[0] != 0) return GDN_ERR_SEQLENS;
    len.resize(n_req);
    for (int32_t r = 0; r < n_req; ++r) {
        if (cu[r + 1] < cu[r]) return GDN_ERR_SEQLENS;
        len[r] = cu[r + 1] - cu[r];
        if (start[r] < 0 || (int64_t)start[r] + len[r] > MAX_ROWS) return GDN_ERR_START;
    }
    return GDN_OK;
}

// A page table: every listed id inside the pool, and enough of them for rows(r) rows of request r.
template <typename F>
int32_t check_table(const attn_pages* p, int32_t n_req, const int32_t* page_cu, const int32_t* page_ids, F rows) {
    if (!page_cu) return GDN_ERR_NULL;
    if (page_cu[0] != 0) return GDN_ERR_SEQLENS;
    for (int32_t r = 0; r < n_req; ++r) {
        if (page_cu[r + 1] < page_cu[r]) return GDN_ERR_SEQLENS;
        if ((int64_t)(page_cu[r + 1] - page_cu[r]) * p->page_rows < rows(r)) return GDN_ERR_START;
    }
    const int32_t n = page_cu[n_req];
    if (n > 0 && !page_ids) return GDN_ERR_NULL;
    bool bad = false;
    for (int32_t i = 0; i < n; ++i) bad |= (uint32_t)page_ids[i] >= (uint32_t)p->n_pages;
    return bad ? GDN_ERR_SLOT_RANGE : GDN_OK;
}

// A set of page ids.
class PageSet {
  public:
    explicit PageSet(int32_t n_pages) : bits_((size_t)n_pages / 64 + 1, 0) {}
    bool has(int32_t id) const { return bits_[(size_t)id / 64] >> (id % 64) & 1; }
    bool add(int32_t id) {       // false: it was there
        const bool was = has(id);
        bits_[(size_t)id / 64] |= 1ull << (id % 64);
        return !was;
    }

  private:
    std::vector<uint64_t> bits_;
};

// The region of the partial results behind the uploaded image: maxima and normalisers, outputs, sums of the unrounded weights.
// attn_key_weights leaves its parts there instead.
inline int64_t part_le_bytes() { return (int64_t)SPLIT_MAX_WGS * ATT_BQ * sizeof(float); }
inline int64_t parts_bytes(int d) {
    return std::max<int64_t>(part_ml_bytes() + part_o_bytes(d) + part_le_bytes(), (int64_t)WGT_PARTS * wgt_keys(d) * sizeof(float));
}
// ints of an image: the page ids, and the attention's plan, or the units of attn_key_weights (at most two tiles of keys to a page of 256 rows, and the
// cut ones), or the arrays of one entry per request of the others
inline int64_t image_bytes(const attn_shape* s, int32_t n_req, int64_t T, int64_t n_ids) {
    const int64_t attend = plan_ints(n_req, T, s->H_q / s->H_kv);
    const int64_t weights = WGT_REC * (2 * n_ids + n_req + WGT_PARTS) + WGT_MERGE * ((int64_t)WGT_PARTS + 1);
    const int64_t ints = std::max<int64_t>(std::max(attend, weights), 8 * (int64_t)n_req + 2) + n_ids;
    return (ints * (int64_t)sizeof(int32_t) + 255) / 256 * 256;
}

int32_t check_workspace(const attn_shape* s, int32_t n_req, int64_t T, int64_t n_ids, const void* ws, int64_t bytes) {
    if (!ws || !aligned16(ws) || bytes < image_bytes(s, n_req, T, n_ids) + parts_bytes(s->d)) return GDN_ERR_WORKSPACE;
    return GDN_OK;
}

// What every call with new tokens checks of its index arrays, in this order.
int32_t check_call(const attn_shape* s, int32_t n_req, const int32_t* cu, const int32_t* start, const attn_pages* pages,
                   const int32_t* page_cu, const int32_t* page_ids, std::vector<int32_t>& len) {
    int32_t rc = check_lengths(n_req, cu, start, len);
    if (rc != GDN_OK) return rc;
    return check_table(pages, n_req, page_cu, page_ids, [&](int32_t r) { return (int64_t)start[r] + len[r]; });
}

int32_t check_front(const attn_shape* s, int32_t n_req, const attn_pages* pages) {
    const int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0) return GDN_ERR_COUNT;
    return check_pages(s, pages);
}

// ---- a call's image to the device.  Small ones go by value (gdn::upload_plan); page tables are larger, and a copy of more than 16 KiB takes the
// stream 20 us between two kernels: these a launch of ours reads out of pinned memory (4 us for 90 KB).  The buffers form a ring; a workgroup that has
// read its piece says so in a word of the buffer, and a call that comes round to a buffer waits (on the host) for all of them.
constexpr int FETCH_RING = 8, FETCH_THREADS = 256, FETCH_PIECE = 16 * FETCH_THREADS;   // bytes per workgroup
constexpr size_t FETCH_ABOVE = 7168;

__global__ void __launch_bounds__(FETCH_THREADS) attn_fetch_kernel(const u32x4* src, u32x4* dst, int64_t n, uint32_t* read, uint32_t mark) {
    const int64_t i = (int64_t)blockIdx.x * FETCH_THREADS + threadIdx.x;
    if (i < n) dst[i] = src[i];
    __syncthreads();                      // (waits for every load of the workgroup, whose values have been stored)
    if (threadIdx.x == 0) __hip_atomic_store(read + blockIdx.x, mark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

struct FetchRing {
    std::mutex mu;
    struct Slot {
        char* host = nullptr;             // words of the workgroups that have read, then the image
        size_t bytes = 0;                 // room for the image
        uint32_t mark = 0, blocks = 0;    // of the last upload
    } slot[FETCH_RING];
    int next = 0;
};
FetchRing g_fetch;

int32_t send_image(const std::vector<int32_t>& img, void* dst, hipStream_t stream) {
    const size_t bytes = img.size() * sizeof(int32_t);
    if (bytes <= FETCH_ABOVE) return gdn::upload_plan(img.data(), bytes, dst, stream);
    std::lock_guard<std::mutex> lock(g_fetch.mu);
    FetchRing::Slot& s = g_fetch.slot[g_fetch.next];
    g_fetch.next = (g_fetch.next + 1) % FETCH_RING;
    const auto words = [](size_t room) { return (room + FETCH_PIECE - 1) / FETCH_PIECE; };
    if (s.host) {
        uint32_t* const read = reinterpret_cast<uint32_t*>(s.host);
        for (uint32_t b = 0; b < s.blocks; ++b)
            while (__atomic_load_n(read + b, __ATOMIC_ACQUIRE) != s.mark) std::this_thread::yield();
    }
    if (s.bytes < bytes) {
        if (s.host) (void)hipHostFree(s.host);
        s.host = nullptr;
        s.bytes = s.blocks = 0;
        const size_t room = (std::max<size_t>(2 * bytes, 1 << 17) + FETCH_PIECE - 1) / FETCH_PIECE * FETCH_PIECE;
        void* p = nullptr;
        const hipError_t e = hipHostMalloc(&p, room + (words(room) * sizeof(uint32_t) + 255) / 256 * 256, hipHostMallocCoherent);
        if (e != hipSuccess) return hip_err(e);
        s.host = static_cast<char*>(p);
        s.bytes = room;
        std::memset(s.host, 0, words(room) * sizeof(uint32_t));
        s.mark = 0;
    }
    uint32_t* const read = reinterpret_cast<uint32_t*>(s.host);
    char* const image = s.host + (words(s.bytes) * sizeof(uint32_t) + 255) / 256 * 256;
    std::memcpy(image, img.data(), bytes);
    const uint32_t blocks = (uint32_t)words(bytes), mark = s.mark + 1 == 0 ? 1 : s.mark + 1;
    hipLaunchKernelGGL(attn_fetch_kernel, dim3(blocks), dim3(FETCH_THREADS), 0, stream, reinterpret_cast<const u32x4*>(image), static_cast<u32x4*>(dst),
                       (int64_t)((bytes + 15) / 16), read, mark);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_err(e);
    s.mark = mark;
    s.blocks = blocks;
    return GDN_OK;
}

// A plan that fits goes by value, with `words` set from it; any other to the workspace.
inline int32_t place_plan(const std::vector<int32_t>& img, PlanWords<true>& words, bool& by_value, void* workspace, hipStream_t stream) {
    by_value = img.size() <= PLAN_WORDS;
    if (!by_value) return send_image(img, workspace, stream);
    std::copy(img.begin(), img.end(), words.w);
    return GDN_OK;
}

int32_t rope_append(const attn_shape* s, const attn_rope* rope, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                    int64_t ldv, int32_t n_req, const int32_t* cu, const int32_t* pos, const int32_t* start, const attn_pages* pages,
                    void* k_pool, void* v_pool, const int32_t* page_cu, const int32_t* page_ids, void* q_out, void* workspace,
                    int64_t workspace_bytes, hipStream_t stream) {
    int32_t rc = check_front(s, n_req, pages);
    if (rc != GDN_OK) return rc;
    if (!rope) return GDN_ERR_NULL;
    if (rope->rot < 0 || rope->rot > s->d || rope->rot % 16 != 0 || (rope->layout != 0 && rope->layout != 1)) return GDN_ERR_SHAPE;
    if (rope->in_dtype != GDN_F32 && rope->in_dtype != GDN_BF16) return GDN_ERR_SHAPE;
    if (!std::isfinite(rope->amplitude)) return GDN_ERR_SHAPE;
    if (rope->rot > 0 && !rope->freq) return GDN_ERR_NULL;
    const int per16 = rope->in_dtype == GDN_F32 ? 4 : 8;
    const int64_t wq = (int64_t)s->H_q * s->d, wkv = (int64_t)s->H_kv * s->d;
    if (ldq % per16 != 0 || ldk % per16 != 0 || ldv % per16 != 0) return GDN_ERR_ALIGN;
    if (ldq < wq || ldk < wkv || ldv < wkv) return GDN_ERR_SHAPE;
    RopeArgs a;
    for (int p = 0; p < rope->rot / 2; ++p) {
        if (!std::isfinite(rope->freq[p])) return GDN_ERR_SHAPE;
        long double t = (long double)rope->freq[p] * 0.159154943091895335768883763372514362L;      // turns: over 2 pi
        if (!(t >= 0.0L && t < 1.0L)) t -= floorl(t);
        t = t * 18446744073709551616.0L + 0.5L;
        a.turn[p] = t >= 18446744073709551616.0L ? 0 : (uint64_t)t;
    }
    if (n_req == 0) return GDN_OK;
    std::vector<int32_t> len;
    rc = check_call(s, n_req, cu, start, pages, page_cu, page_ids, len);
    if (rc != GDN_OK) return rc;
    if (!pos) pos = start;
    for (int32_t r = 0; r < n_req; ++r)
        if (pos[r] < 0 || (int64_t)pos[r] + len[r] > INT32_MAX) return GDN_ERR_START;
    const int64_t T = cu[n_req];
    if (T == 0) return GDN_OK;
    // ---- the pages that get rows, and that nobody else in the call has them
    const int shift = shift_of(pages);
    std::vector<int32_t> img((size_t)(4 * (int64_t)n_req + 1));
    PageSet written(pages->n_pages);
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t p0 = start[r] >> shift;
        img[1 + n_req + r] = start[r];
        img[1 + 2 * n_req + r] = pos[r];
        img[1 + 3 * n_req + r] = (int32_t)(img.size() - (4 * (size_t)n_req + 1)) - p0;
        if (len[r] == 0) continue;
        const int32_t p1 = (start[r] + len[r] - 1) >> shift;
        for (int32_t p = p0; p <= p1; ++p) {
            if (!written.add(page_ids[page_cu[r] + p])) return GDN_ERR_SLOT_DUP;
            img.push_back(page_ids[page_cu[r] + p]);
        }
    }
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t held = (start[r] + (1 << shift) - 1) >> shift, p0 = len[r] > 0 ? start[r] >> shift : held;
        for (int32_t p = 0; p < p0; ++p)
            if (written.has(page_ids[page_cu[r] + p])) return GDN_ERR_SLOT_DUP;
    }
    for (int32_t r = 0; r <= n_req; ++r) img[r] = cu[r];
    if (!q || !k || !v || !k_pool || !v_pool || !q_out) return GDN_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(q_out)) return GDN_ERR_ALIGN;
    rc = check_workspace(s, n_req, T, page_cu[n_req], workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;
    PlanWords<true> words;
    bool by_value;
    rc = place_plan(img, words, by_value, workspace, stream);
    if (rc != GDN_OK) return rc;
    a.q = q; a.k = k; a.v = v;
    a.q_out = static_cast<uint16_t*>(q_out);
    a.k_pool = static_cast<uint16_t*>(k_pool);
    a.v_pool = static_cast<uint16_t*>(v_pool);
    a.plan = static_cast<const int32_t*>(workspace);
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.page_stride = pages->page_stride;
    a.n_req = n_req;
    a.T = (int32_t)T;
    // as many tokens to a workgroup as its threads have on their way at once, but one while there are fewer tokens than compute units
    const int64_t units = ((int64_t)s->H_q + 2 * s->H_kv) * (s->d / 16);
    a.tokens = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(int64_t)ROPE_TOKENS, ROPE_UNITS * ROPE_THREADS / units, (T + 255) / 256}));
    if (units * ROPE_TOKENS > INT32_MAX) return GDN_ERR_SHAPE;
    a.H_q = s->H_q; a.H_kv = s->H_kv;
    a.unit_shift = __builtin_ctz((unsigned)s->d / 16);
    a.page_shift = shift;
    a.rot = rope->rot;
    a.layout = rope->layout;
    a.amplitude = rope->amplitude;
    const dim3 grid((unsigned)((T + a.tokens - 1) / a.tokens)), block(ROPE_THREADS);
    const bool f32 = rope->in_dtype == GDN_F32;
    if (by_value && f32) hipLaunchKernelGGL((attn_rope_kernel<true, true>), grid, block, 0, stream, a, words);
    else if (by_value) hipLaunchKernelGGL((attn_rope_kernel<false, true>), grid, block, 0, stream, a, words);
    else if (f32) hipLaunchKernelGGL((attn_rope_kernel<true, false>), grid, block, 0, stream, a, PlanWords<false>());
    else hipLaunchKernelGGL((attn_rope_kernel<false, false>), grid, block, 0, stream, a, PlanWords<false>());
    return hip_err(hipGetLastError());
}

template <bool LSE>
int32_t launch_paged(const attn_shape* s, const UnitPlan& plan, const CallImage& im, const int32_t* d, bool nt, PagedArgs& a, hipStream_t stream) {
    int32_t rc;
    if (im.n_narrow > 0 && (rc = launch_narrow_units<LSE>(s, nt, im, a, stream)) != GDN_OK) return rc;
    if (im.n_wide > 0 && (rc = launch_wide_units<LSE>(s, plan, im, a, stream)) != GDN_OK) return rc;
    return launch_merge<LSE, true>(s, plan, im, d, a, a.lse, a.part_le, stream);
}

int32_t paged_prefill(const attn_shape* s, const void* q, const void* gate, int32_t n_req, const int32_t* cu, const int32_t* start,
                      const attn_pages* pages, const void* k_pool, const void* v_pool, const int32_t* page_cu, const int32_t* page_ids,
                      void* o, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    int32_t rc = check_front(s, n_req, pages);
    if (rc != GDN_OK) return rc;
    if (n_req == 0) return GDN_OK;
    std::vector<int32_t> len;
    rc = check_call(s, n_req, cu, start, pages, page_cu, page_ids, len);
    if (rc != GDN_OK) return rc;
    const int64_t T = cu[n_req];
    if (T == 0) return GDN_OK;
    if (!q || !k_pool || !v_pool || !o) return GDN_ERR_NULL;
    if (!aligned16(q) || !aligned16(gate) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(o)) return GDN_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0) return GDN_ERR_ALIGN;
    const int32_t n_ids = page_cu[n_req];
    rc = check_workspace(s, n_req, T, n_ids, workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;

    UnitPlan plan;
    build_units(*s, n_req, len.data(), start, plan);
    CallImage im;
    rc = make_image(s, plan, n_req, cu, start, len.data(), page_cu, page_ids, n_ids, im);
    if (rc != GDN_OK) return rc;
    rc = send_image(im.img, workspace, stream);
    if (rc != GDN_OK) return rc;
    const int32_t* const d = static_cast<const int32_t*>(workspace);
    char* const parts = static_cast<char*>(workspace) + image_bytes(s, n_req, T, n_ids);
    PagedArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.gate = static_cast<const uint16_t*>(gate);
    a.k_cache = static_cast<const uint16_t*>(k_pool);
    a.v_cache = static_cast<const uint16_t*>(v_pool);
    a.o = o;
    a.slot_stride = pages->page_stride;
    image_args(s, plan, n_req, im, d, parts, a);
    a.page_ids = d + im.ids_at;
    a.page_shift = shift_of(pages);
    a.lse = lse;
    a.part_le = reinterpret_cast<float*>(parts + part_ml_bytes() + part_o_bytes(s->d));
    const bool nt = narrow_nt(s, plan, n_req, start, len.data());
    return lse ? launch_paged<true>(s, plan, im, d, nt, a, stream) : launch_paged<false>(s, plan, im, d, nt, a, stream);
}

template <int D, bool BY_VALUE>
void launch_weights_d(bool few, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    if (few) hipLaunchKernelGGL((attn_weights_few_kernel<D, BY_VALUE>), dim3(blocks), dim3(WGT_THREADS), 0, stream, a, words);
    else hipLaunchKernelGGL((attn_weights_kernel<D, BY_VALUE>), dim3(blocks), dim3(WGT_THREADS), 0, stream, a, words);
}
template <bool BY_VALUE>
void launch_weights(int d, bool few, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    switch (d) {
        case 64: launch_weights_d<64>(few, a, words, blocks, stream); break;
        case 128: launch_weights_d<128>(few, a, words, blocks, stream); break;
        default: launch_weights_d<256>(few, a, words, blocks, stream); break;
    }
}
template <bool BY_VALUE>
void launch_weights_merge(int d, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    const dim3 block((unsigned)wgt_keys(d));
    if (d == 256) hipLaunchKernelGGL((attn_weights_merge_kernel<wgt_keys(256), BY_VALUE>), dim3(blocks), block, 0, stream, a, words);
    else hipLaunchKernelGGL((attn_weights_merge_kernel<wgt_keys(128), BY_VALUE>), dim3(blocks), block, 0, stream, a, words);
}

// The work of one attn_key_weights call: units (a tile of keys and a run of the request's query rows) of either kernel, and the tiles whose rows are cut.
struct WeightPlan {
    std::vector<int32_t> wide, few, merge;       // WGT_REC, WGT_REC, WGT_MERGE ints each
};

// The rows of a tile are cut on a grid of `run` row tiles of 64, the first quarter of them four times finer, so that the chip is full and the short units,
// which go last, fill its end: a workgroup takes as long as its row tiles and about WGT_START more for its keys, and WGT_SLOTS of them run at
// once (two to a compute unit).
constexpr int WGT_SLOTS = 512, WGT_START = 2;
struct RowGrid {
    int64_t run, fine, edge;             // row tiles per cut behind `edge` and before it (a multiple of `fine`)
    RowGrid(int64_t run, int64_t m) : run(run), fine(std::max<int64_t>(1, run / 4)), edge(run >= m ? 0 : m / 4 / fine * fine) {}
    int64_t index(int64_t tile) const { return tile < edge ? tile / fine : edge / fine + (tile - edge) / run; }
    int64_t begin(int64_t i) const { return i < edge / fine ? i * fine : edge + (i - edge / fine) * run; }
};

void plan_weights(const attn_shape* s, int32_t n_req, const int32_t* cu, const int32_t* start, const int32_t* len, const int32_t* place, WeightPlan& out) {
    const int G = s->H_q / s->H_kv, keys = wgt_keys(s->d);
    auto is_few = [&](int32_t r) { return len[r] > 0 && (int64_t)len[r] * G <= WGT_FEW; };
    auto tiles_of = [&](int32_t r) { return (int32_t)(((int64_t)start[r] + len[r] + keys - 1) / keys); };
    auto row_tiles = [&](int32_t r) { return (int32_t)(((int64_t)len[r] * G + WGT_ROWS - 1) / WGT_ROWS); };
    auto first_seen = [&](int32_t r, int32_t tile) {       // the first row tile that sees a key of the tile
        return (int32_t)(std::max<int64_t>(0, (int64_t)tile * keys - start[r]) * G / WGT_ROWS);
    };
    // ---- units and row tiles in all if rows are cut every `run` row tiles
    int64_t work = 0, most = 0;
    auto units_of = [&](int64_t run, int64_t& cut) {
        int64_t units = 0;
        cut = work = 0;
        for (int32_t r = 0; r < n_req; ++r) {
            if (is_few(r)) continue;
            const int64_t m = row_tiles(r);
            most = std::max(most, m);
            const RowGrid grid(run, m);
            const int64_t whole = std::min<int64_t>(tiles_of(r), start[r] / keys + 1), parts = m > 0 ? grid.index(m - 1) + 1 : 1;   // tiles that every row sees a key of
            units += whole * parts;
            work += whole * m;
            if (parts > 1) cut += whole * parts;
            for (int32_t t = (int32_t)whole; t < tiles_of(r); ++t) {
                const int64_t f = first_seen(r, t), p = grid.index(m - 1) - grid.index(f) + 1;
                units += p;
                work += m - f;
                if (p > 1) cut += p;
            }
        }
        return units;
    };
    int64_t cut = 0, units = units_of(INT32_MAX, cut), run = std::max<int64_t>(most, 1);
    if (most > 1) {
        auto cost = [&](int64_t c, int64_t n) {            // units that fill every gap but half of the last short one, and no less than one unit
            const int64_t last = c < most ? std::max<int64_t>(1, c / 4) : c;
            const double even = (double)((work + WGT_START * n) * s->H_kv) / WGT_SLOTS + 0.5 * (double)(last + WGT_START);
            return std::max(even, (double)(c + WGT_START));
        };
        double best = cost(most, units);
        for (int64_t c = most; c > 1;) {
            c = c > 8 ? c * 3 / 4 : c - 1;
            const int64_t n = units_of(c, cut);
            if (cut * s->H_kv > WGT_PARTS) break;
            if (cost(c, n) < 0.97 * best) {
                best = cost(c, n);
                run = c;
                units = n;
            }
        }
    }
    // ---- the units, those of the same rows together (they read the same queries), the longest first
    struct Unit { int32_t r, kv0, lo, hi, part; };
    std::vector<Unit> list;
    list.reserve((size_t)units);
    std::vector<int32_t> base;
    int32_t slot = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t tiles = tiles_of(r);
        if (is_few(r)) {
            for (int32_t t = 0; t < tiles; ++t)
                out.few.insert(out.few.end(), {cu[r], len[r], start[r], place[r], t * keys, 0, len[r] * G, -1});
            continue;
        }
        const int32_t m = row_tiles(r), rows = len[r] * G;
        if (m == 0) {
            for (int32_t t = 0; t < tiles; ++t) list.push_back({r, t * keys, 0, 0, -1});
            continue;
        }
        base.resize(tiles);
        const RowGrid grid(run, m);
        auto cut_of = [&](int32_t t) { return (int32_t)grid.index(first_seen(r, t)); };      // the first cut of rows that sees a key of tile t
        const int32_t cuts = (int32_t)grid.index(m - 1) + 1;
        for (int32_t t = 0; t < tiles; ++t) {
            const int32_t parts = cuts - cut_of(t);
            base[t] = slot - cut_of(t);                  // + the cut's number: its partial sum
            if (parts <= 1) continue;
            out.merge.insert(out.merge.end(), {start[r] + len[r], start[r], place[r], t * keys, slot});
            slot += parts;
        }
        for (int32_t c = cuts - 1; c >= 0; --c) {
            const int32_t lo = (int32_t)grid.begin(c), hi = (int32_t)std::min<int64_t>(grid.begin(c + 1), m);
            for (int32_t t = 0; t < tiles; ++t) {
                const int32_t f = std::max(lo, first_seen(r, t));
                if (f >= hi) break;
                list.push_back({r, t * keys, f * WGT_ROWS, std::min(hi * WGT_ROWS, rows), cuts - cut_of(t) <= 1 ? -1 : base[t] + c});
            }
        }
    }
    if (!out.merge.empty()) out.merge.insert(out.merge.end(), {0, 0, 0, 0, slot});
    // by length, in classes: a counting sort that keeps their order
    constexpr int CLASSES = 64;
    const int64_t top = std::max<int64_t>(1, std::min<int64_t>(run, most)) * WGT_ROWS;
    std::vector<int32_t> at(CLASSES + 1, 0);
    auto class_of = [&](const Unit& u) { return (int)(CLASSES - 1 - (int64_t)(u.hi - u.lo) * (CLASSES - 1) / top); };
    for (const Unit& u : list) ++at[class_of(u) + 1];
    for (int i = 0; i < CLASSES; ++i) at[i + 1] += at[i];
    out.wide.resize(list.size() * WGT_REC);
    for (const Unit& u : list) {
        int32_t* const rec = out.wide.data() + (size_t)at[class_of(u)]++ * WGT_REC;
        const int32_t x[WGT_REC] = {cu[u.r], len[u.r], start[u.r], place[u.r], u.kv0, u.lo, u.hi, u.part};
        std::copy(x, x + WGT_REC, rec);
    }
}

int32_t key_weights(const attn_shape* s, const void* q, const float* lse, int32_t n_req, const int32_t* cu, const int32_t* start,
                    const attn_pages* pages, const void* k_pool, const int32_t* page_cu, const int32_t* page_ids, float decay,
                    const float* w_in, float* w_out, int64_t w_stride, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    int32_t rc = check_front(s, n_req, pages);
    if (rc != GDN_OK) return rc;
    if (!std::isfinite(decay) || w_stride < (int64_t)s->H_kv * pages->page_rows) return GDN_ERR_SHAPE;
    if (n_req == 0) return GDN_OK;
    std::vector<int32_t> len;
    rc = check_call(s, n_req, cu, start, pages, page_cu, page_ids, len);
    if (rc != GDN_OK) return rc;
    const int shift = shift_of(pages);
    PageSet written(pages->n_pages);
    int64_t rows = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t total = start[r] + len[r];
        rows += total;
        for (int32_t p = 0; (int64_t)p << shift < total; ++p)
            if (!written.add(page_ids[page_cu[r] + p])) return GDN_ERR_SLOT_DUP;
    }
    if (rows == 0) return GDN_OK;
    const int64_t T = cu[n_req];
    if ((T > 0 && (!q || !lse)) || !k_pool || !w_out) return GDN_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_pool)) return GDN_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0 || reinterpret_cast<uintptr_t>(w_in) % 4 != 0 || reinterpret_cast<uintptr_t>(w_out) % 4 != 0) return GDN_ERR_ALIGN;
    const int32_t n_ids = page_cu[n_req];
    rc = check_workspace(s, n_req, T, n_ids, workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;

    const int G = s->H_q / s->H_kv;
    for (int32_t r = 0; r < n_req; ++r)
        if (((int64_t)len[r] + 512) * G > INT32_MAX) return GDN_ERR_SHAPE;
    if (((int64_t)s->H_q * (WGT_ROWS + 1) + G) * s->d * 2 > INT32_MAX) return GDN_ERR_SHAPE;
    WeightPlan plan;
    plan_weights(s, n_req, cu, start, len.data(), page_cu, plan);
    const int64_t n_wide = (int64_t)plan.wide.size() / WGT_REC, n_few = (int64_t)plan.few.size() / WGT_REC;
    const int64_t n_cut = plan.merge.empty() ? 0 : (int64_t)plan.merge.size() / WGT_MERGE - 1;
    if (std::max(n_wide, n_few) * s->H_kv > INT32_MAX) return GDN_ERR_COUNT;
    std::vector<int32_t> img(plan.wide.size() + plan.few.size() + plan.merge.size() + (size_t)n_ids);
    const int64_t few_at = (int64_t)plan.wide.size(), merge_at = few_at + (int64_t)plan.few.size(), ids_at = merge_at + (int64_t)plan.merge.size();
    std::copy(plan.wide.begin(), plan.wide.end(), img.begin());
    std::copy(plan.few.begin(), plan.few.end(), img.begin() + few_at);
    std::copy(plan.merge.begin(), plan.merge.end(), img.begin() + merge_at);
    std::copy(page_ids, page_ids + n_ids, img.begin() + ids_at);
    PlanWords<true> words;
    bool by_value;
    rc = place_plan(img, words, by_value, workspace, stream);
    if (rc != GDN_OK) return rc;
    WeightArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.lse = lse;
    a.k_pool = static_cast<const uint16_t*>(k_pool);
    a.w_in = w_in;
    a.w_out = w_out;
    a.plan = static_cast<const int32_t*>(workspace);
    a.merges = (int32_t)merge_at;
    a.ids = (int32_t)ids_at;
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + image_bytes(s, n_req, T, n_ids));
    a.page_stride = pages->page_stride;
    a.w_stride = w_stride;
    a.H_q = s->H_q; a.H_kv = s->H_kv; a.G = G;
    a.page_shift = shift;
    a.inv_G = 1.f / (float)G;
    a.scale_log2e = s->scale * 1.4426950408889634f;
    a.decay = decay;
    auto launch = [&](const auto& words) {
        hipError_t e = hipSuccess;
        if (n_few > 0) {
            a.units = (int32_t)few_at;
            launch_weights(s->d, true, a, words, (unsigned)(n_few * s->H_kv), stream);
            e = hipGetLastError();
        }
        if (e == hipSuccess && n_wide > 0) {
            a.units = 0;
            launch_weights(s->d, false, a, words, (unsigned)(n_wide * s->H_kv), stream);
            e = hipGetLastError();
        }
        if (e == hipSuccess && n_cut > 0) {
            launch_weights_merge(s->d, a, words, (unsigned)(n_cut * s->H_kv), stream);
            e = hipGetLastError();
        }
        return hip_err(e);
    };
    return by_value ? launch(words) : launch(PlanWords<false>());
}

template <int D, bool BY_VALUE>
void launch_gather(const EvictArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    hipLaunchKernelGGL((attn_gather_rows_kernel<D, BY_VALUE>), dim3(blocks), dim3(GATHER_THREADS), 0, stream, a, words);
}

int32_t evict(const attn_shape* s, int32_t n_req, const int32_t* rows, const int32_t* keep, const int32_t* first, const int32_t* recent,
              const attn_pages* pages, void* k_pool, void* v_pool, float* w_pool, int64_t w_stride, const int32_t* page_cu,
              const int32_t* page_ids, const int32_t* new_page_cu, const int32_t* new_page_ids, int32_t* index, void* workspace,
              int64_t workspace_bytes, hipStream_t stream) {
    int32_t rc = check_front(s, n_req, pages);
    if (rc != GDN_OK) return rc;
    if (w_stride < (int64_t)s->H_kv * pages->page_rows) return GDN_ERR_SHAPE;
    if (n_req == 0) return GDN_OK;
    if (!rows || !keep || !first || !recent) return GDN_ERR_NULL;
    std::vector<int32_t> kept(n_req);
    int64_t total = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        if (rows[r] < 0 || keep[r] < 0 || first[r] < 0 || recent[r] < 0 || rows[r] > MAX_ROWS) return GDN_ERR_START;
        kept[r] = std::min(keep[r], rows[r]);
        if ((int64_t)first[r] + recent[r] > kept[r]) return GDN_ERR_START;
        total += kept[r];
    }
    if (total * s->H_kv > INT32_MAX) return GDN_ERR_COUNT;
    rc = check_table(pages, n_req, page_cu, page_ids, [&](int32_t r) { return (int64_t)rows[r]; });
    if (rc != GDN_OK) return rc;
    rc = check_table(pages, n_req, new_page_cu, new_page_ids, [&](int32_t r) { return (int64_t)kept[r]; });
    if (rc != GDN_OK) return rc;
    const int32_t n_old = page_cu[n_req], n_new = new_page_cu[n_req];
    PageSet fresh(pages->n_pages);
    for (int32_t i = 0; i < n_new; ++i)
        if (!fresh.add(new_page_ids[i])) return GDN_ERR_SLOT_DUP;
    for (int32_t i = 0; i < n_old; ++i)
        if (fresh.has(page_ids[i])) return GDN_ERR_SLOT_HAZARD;
    if (total == 0) return GDN_OK;
    if (!k_pool || !v_pool || !w_pool || !index) return GDN_ERR_NULL;
    if (!aligned16(k_pool) || !aligned16(v_pool)) return GDN_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(w_pool) % 4 != 0 || reinterpret_cast<uintptr_t>(index) % 4 != 0) return GDN_ERR_ALIGN;
    rc = check_workspace(s, n_req, 0, (int64_t)n_old + n_new, workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;

    const int copied = gather_rows(s->d);              // rows per workgroup of the copy
    std::vector<int32_t> img((size_t)(8 * (int64_t)n_req + 2 + n_old + n_new));
    int32_t* p = img.data();
    p = std::copy(rows, rows + n_req, p);
    p = std::copy(kept.begin(), kept.end(), p);
    p = std::copy(first, first + n_req, p);
    p = std::copy(recent, recent + n_req, p);
    p = std::copy(page_cu, page_cu + n_req, p);
    for (int32_t r = 0; r < n_req; ++r) *p++ = n_old + new_page_cu[r];
    *p++ = 0;
    for (int32_t r = 0; r < n_req; ++r, ++p) *p = p[-1] + kept[r];
    *p++ = 0;
    for (int32_t r = 0; r < n_req; ++r, ++p) *p = p[-1] + (kept[r] + copied - 1) / copied;
    const int64_t blocks = (int64_t)p[-1] * s->H_kv;
    p = std::copy(page_ids, page_ids + n_old, p);
    p = std::copy(new_page_ids, new_page_ids + n_new, p);
    if (blocks > INT32_MAX || (int64_t)n_req * s->H_kv > INT32_MAX) return GDN_ERR_COUNT;
    PlanWords<true> words;
    bool by_value;
    rc = place_plan(img, words, by_value, workspace, stream);
    if (rc != GDN_OK) return rc;
    EvictArgs a;
    a.k_pool = static_cast<uint16_t*>(k_pool);
    a.v_pool = static_cast<uint16_t*>(v_pool);
    a.w_pool = w_pool;
    a.index = index;
    a.plan = static_cast<const int32_t*>(workspace);
    a.page_stride = pages->page_stride;
    a.w_stride = w_stride;
    a.n_req = n_req;
    a.H_kv = s->H_kv;
    a.page_shift = shift_of(pages);
    auto launch = [&](const auto& words) {
        constexpr bool BY_VALUE = std::is_same<std::decay_t<decltype(words)>, PlanWords<true>>::value;
        hipLaunchKernelGGL((attn_select_kernel<BY_VALUE>), dim3((unsigned)(n_req * s->H_kv)), dim3(SEL_THREADS), 0, stream, a, words);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_err(e);
        switch (s->d) {
            case 64: launch_gather<64>(a, words, (unsigned)blocks, stream); break;
            case 128: launch_gather<128>(a, words, (unsigned)blocks, stream); break;
            default: launch_gather<256>(a, words, (unsigned)blocks, stream); break;
        }
        return hip_err(hipGetLastError());
    };
    return by_value ? launch(words) : launch(PlanWords<false>());
}

// No exception leaves a C entry: host memory that runs out is a count too large.
template <typename F>
int32_t guarded(F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return GDN_ERR_COUNT;
    } catch (const std::length_error&) {
        return GDN_ERR_COUNT;
    }
}

}  // namespace
}  // namespace attn

using namespace attn;

extern "C" {

int32_t attn_rope_freqs(int32_t rot, double base, int32_t kind, double factor, double context, double fast, double slow, double* freq,
                        double* amplitude) {
    if (!amplitude || (rot > 0 && !freq)) return GDN_ERR_NULL;
    if (rot < 0 || rot % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return GDN_ERR_SHAPE;
    if (kind < ATTN_ROPE_PLAIN || kind > ATTN_ROPE_RAMP) return GDN_ERR_SHAPE;
    if (kind != ATTN_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return GDN_ERR_SHAPE;
    if (kind == ATTN_ROPE_BASE && rot == 2) return GDN_ERR_SHAPE;
    *amplitude = 1.0;
    double lo = 0.0, hi = 0.0;
    if (kind == ATTN_ROPE_RAMP) {
        if (!(context > 0.0 && std::isfinite(context) && slow > 0.0 && fast > slow && std::isfinite(fast))) return GDN_ERR_SHAPE;
        *amplitude = 0.1 * std::log(factor) + 1.0;
        // the pair (a real number) that makes `turns` turns over the context
        auto at = [&](double turns) { return rot * std::log(context / (turns * 6.283185307179586)) / (2.0 * std::log(base)); };
        lo = std::max(std::floor(at(fast)), 0.0);
        hi = std::min(std::ceil(at(slow)), (double)rot - 1.0);
    }
    if (kind == ATTN_ROPE_BASE && rot > 2) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int32_t p = 0; p < rot / 2; ++p) {
        double f = std::pow(base, -2.0 * p / rot);
        if (kind == ATTN_ROPE_LINEAR) f /= factor;
        if (kind == ATTN_ROPE_RAMP) {
            const double w = std::min(std::max((p - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
            f = f * (1.0 - w) + f / factor * w;
        }
        freq[p] = f;
    }
    return GDN_OK;
}

int64_t attn_paged_workspace_bytes(const attn_shape* s, int32_t n_req, int64_t total_tokens, int64_t n_page_ids) {
    const int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0 || total_tokens < 0 || total_tokens > INT32_MAX || n_page_ids < 0 || n_page_ids > 2 * (int64_t)INT32_MAX) return GDN_ERR_COUNT;
    return image_bytes(s, n_req, total_tokens, n_page_ids) + parts_bytes(s->d);
}

int32_t attn_rope_append(const attn_shape* s, const attn_rope* rope, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                         int64_t ldv, int32_t n_req, const int32_t* cu_seqlens, const int32_t* pos, const int32_t* start,
                         const attn_pages* pages, void* k_pool, void* v_pool, const int32_t* page_cu, const int32_t* page_ids, void* q_out,
                         void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] {
        return rope_append(s, rope, q, ldq, k, ldk, v, ldv, n_req, cu_seqlens, pos, start, pages, k_pool, v_pool, page_cu, page_ids, q_out,
                           workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    });
}

int32_t attn_paged_prefill(const attn_shape* s, const void* q, const void* out_gate, int32_t n_req, const int32_t* cu_seqlens,
                           const int32_t* start, const attn_pages* pages, const void* k_pool, const void* v_pool, const int32_t* page_cu,
                           const int32_t* page_ids, void* o, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] {
        return paged_prefill(s, q, out_gate, n_req, cu_seqlens, start, pages, k_pool, v_pool, page_cu, page_ids, o, lse, workspace,
                             workspace_bytes, static_cast<hipStream_t>(stream));
    });
}

int32_t attn_key_weights(const attn_shape* s, const void* q, const float* lse, int32_t n_req, const int32_t* cu_seqlens,
                         const int32_t* start, const attn_pages* pages, const void* k_pool, const int32_t* page_cu, const int32_t* page_ids,
                         float decay, const float* w_in, float* w_out, int64_t w_stride, void* workspace, int64_t workspace_bytes,
                         void* stream) {
    return guarded([&] {
        return key_weights(s, q, lse, n_req, cu_seqlens, start, pages, k_pool, page_cu, page_ids, decay, w_in, w_out, w_stride, workspace,
                           workspace_bytes, static_cast<hipStream_t>(stream));
    });
}

int32_t attn_evict(const attn_shape* s, int32_t n_req, const int32_t* rows, const int32_t* keep, const int32_t* first,
                   const int32_t* recent, const attn_pages* pages, void* k_pool, void* v_pool, float* w_pool, int64_t w_stride,
                   const int32_t* page_cu, const int32_t* page_ids, const int32_t* new_page_cu, const int32_t* new_page_ids, int32_t* index,
                   void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] {
        return evict(s, n_req, rows, keep, first, recent, pages, k_pool, v_pool, w_pool, w_stride, page_cu, page_ids, new_page_cu,
                     new_page_ids, index, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
