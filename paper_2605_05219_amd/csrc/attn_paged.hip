// attn_paged: host side of the paged key/value cache (see include/attn_paged.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <chrono>
#include <cmath>
#include <mutex>
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

// The lengths of a page table: enough pages listed for rows(r) rows of request r.
template <typename F>
int32_t check_table(const attn_pages* p, int32_t n_req, const int32_t* page_cu, const int32_t* page_ids, F rows) {
    if (!page_cu) return GDN_ERR_NULL;
    if (page_cu[0] != 0) return GDN_ERR_SEQLENS;
    for (int32_t r = 0; r < n_req; ++r) {
        if (page_cu[r + 1] < page_cu[r]) return GDN_ERR_SEQLENS;
        if ((int64_t)(page_cu[r + 1] - page_cu[r]) * p->page_rows < rows(r)) return GDN_ERR_START;
    }
    return page_cu[n_req] > 0 && !page_ids ? GDN_ERR_NULL : GDN_OK;
}

// Its ids, all inside the pool.
int32_t check_ids(const attn_pages* p, const int32_t* ids, int64_t n) {
    uint32_t bad = 0;
    for (int64_t i = 0; i < n; ++i) bad |= (uint32_t)ids[i] >= (uint32_t)p->n_pages;
    return bad ? GDN_ERR_SLOT_RANGE : GDN_OK;
}

// A set of page ids.  The bits are the thread's own between calls (a long table would cost the calls fresh memory each time).
class PageSet {
  public:
    explicit PageSet(int32_t n_pages) {
        thread_local std::vector<uint64_t> store;
        bits_ = &store;
        store.assign((size_t)n_pages / 64 + 1, 0);
    }
    bool has(int32_t id) const { return (*bits_)[(size_t)id / 64] >> (id % 64) & 1; }
    // ids inside the pool; false: one of them was there
    bool add(const int32_t* ids, int64_t n) {
        uint64_t* const b = bits_->data();
        uint64_t twice = 0;
        for (int64_t i = 0; i < n; ++i) {
            uint64_t& word = b[(uint32_t)ids[i] / 64];
            const uint64_t bit = 1ull << ((uint32_t)ids[i] % 64);
            twice |= word & bit;
            word |= bit;
        }
        return twice == 0;
    }

  private:
    std::vector<uint64_t>* bits_;
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
int32_t check_call(int32_t n_req, const int32_t* cu, const int32_t* start, const attn_pages* pages,
                   const int32_t* page_cu, const int32_t* page_ids, std::vector<int32_t>& len) {
    int32_t rc = check_lengths(n_req, cu, start, len);
    if (rc != GDN_OK) return rc;
    rc = check_table(pages, n_req, page_cu, page_ids, [&](int32_t r) { return (int64_t)start[r] + len[r]; });
    return rc != GDN_OK ? rc : check_ids(pages, page_ids, page_cu[n_req]);
}

int32_t check_front(const attn_shape* s, int32_t n_req, const attn_pages* pages) {
    const int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0) return GDN_ERR_COUNT;
    return check_pages(s, pages);
}

// ---- a call's plan (its index arrays) to the device.  Up to PLAN_WORDS go by value, in the arguments of the call's launches, and up to SMALL_WORDS in those
// of a small launch (gdn::write_plan).  Longer page tables cost more: a copy of more than 16 KiB takes the stream 20 us between two kernels.  These
// are written into pinned memory, out of which a launch of ours reads them (4 us for 90 KB).  The buffers are the process's; a workgroup that has read
// its piece says so in a word of the buffer, and a buffer is free when all of them have.  Where none is, a call waits (on the host, with no lock held)
// for FETCH_PATIENCE at most: calls in a row on a busy stream stay that close to the device.  Behind that its plan goes by value, in small launches (26 for
// 90 KB), so that a stream that stands still, or a device that has failed, holds up no call on another one.  A graph's replay would read
// what a later call wrote to a buffer, and its capture reads nothing that the wait could see: such a call under capture is refused.
constexpr int FETCH_RING = 8, FETCH_THREADS = 256, FETCH_PIECE = 16 * FETCH_THREADS;   // bytes per workgroup
constexpr std::chrono::microseconds FETCH_PATIENCE(2000);
constexpr int SMALL_WORDS = 1792;

__global__ void __launch_bounds__(FETCH_THREADS) attn_fetch_kernel(const u32x4* src, u32x4* dst, int64_t n, uint32_t* read, uint32_t mark) {
    const int64_t i = (int64_t)blockIdx.x * FETCH_THREADS + threadIdx.x;
    if (i < n) dst[i] = src[i];
    __syncthreads();                      // (waits for every load of the workgroup, whose values have been stored)
    if (threadIdx.x == 0) __hip_atomic_store(read + blockIdx.x, mark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

class FetchRing {
  public:
    struct Slot {
        char* host = nullptr;             // words of the workgroups that have read, then the plan
        size_t bytes = 0;                 // room for the plan
        uint32_t mark = 0, blocks = 0;    // of the last upload
        bool taken = false;               // a call is writing it
        size_t words_bytes() const { return (bytes / FETCH_PIECE * sizeof(uint32_t) + 255) / 256 * 256; }
        bool read() const {
            const uint32_t* const words = reinterpret_cast<const uint32_t*>(host);
            for (uint32_t b = 0; b < blocks; ++b)
                if (__atomic_load_n(words + b, __ATOMIC_ACQUIRE) != mark) return false;
            return true;
        }
    };
    // A free buffer, the caller's until it is given back, or nullptr.
    Slot* take() {
        std::lock_guard<std::mutex> lock(mu_);
        for (int i = 0; i < FETCH_RING; ++i) {
            Slot& s = slot_[(next_ + i) % FETCH_RING];
            if (s.taken || !s.read()) continue;
            s.taken = true;
            next_ = (next_ + i + 1) % FETCH_RING;
            return &s;
        }
        return nullptr;
    }
    void give_back(Slot* s) {
        std::lock_guard<std::mutex> lock(mu_);
        s->taken = false;
    }

  private:
    std::mutex mu_;                       // held to look at the slots, not to wait or to write them
    Slot slot_[FETCH_RING];
    int next_ = 0;
};
FetchRing g_fetch;

class Plan {
  public:
    Plan() = default;
    Plan(const Plan&) = delete;
    Plan& operator=(const Plan&) = delete;
    ~Plan() {
        if (slot_) g_fetch.give_back(slot_);
    }
    // Room for `ints` words at data(); up to PLAN_WORDS of them go by value.
    int32_t open(int64_t ints, hipStream_t stream) {
        ints_ = ints;
        by_value_ = ints <= PLAN_WORDS;
        if (ints <= SMALL_WORDS) {
            data_ = by_value_ ? arguments_.w : small_.w;
            return GDN_OK;
        }
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        const hipError_t asked = hipStreamIsCapturing(stream, &capture);
        if (asked != hipSuccess) return hip_err(asked);
        if (capture != hipStreamCaptureStatusNone) return hip_err(hipErrorStreamCaptureUnsupported);
        slot_ = g_fetch.take();
        if (!slot_) {
            const auto until = std::chrono::steady_clock::now() + FETCH_PATIENCE;
            while (!(slot_ = g_fetch.take()) && std::chrono::steady_clock::now() < until) std::this_thread::yield();
        }
        if (!slot_) {
            long_.resize((size_t)ints);
            data_ = long_.data();
            return GDN_OK;
        }
        FetchRing::Slot& s = *slot_;
        const size_t bytes = (size_t)ints * sizeof(int32_t);
        if (s.bytes < bytes) {            // (a buffer outgrown is not freed, which would wait for the device: the next one is more than twice as long)
            FetchRing::Slot fresh;
            fresh.bytes = (std::max<size_t>(2 * bytes, 1 << 17) + FETCH_PIECE - 1) / FETCH_PIECE * FETCH_PIECE;
            void* p = nullptr;
            const hipError_t e = hipHostMalloc(&p, fresh.bytes + fresh.words_bytes(), hipHostMallocCoherent | hipHostMallocPortable);
            if (e != hipSuccess) return hip_err(e);
            std::memset(p, 0, fresh.words_bytes());
            s.host = static_cast<char*>(p);      // (`taken` is the lock's)
            s.bytes = fresh.bytes;
            s.mark = s.blocks = 0;
        }
        data_ = reinterpret_cast<int32_t*>(s.host + s.words_bytes());
        return GDN_OK;
    }
    int32_t* data() { return data_; }
    bool by_value() const { return by_value_; }
    const PlanWords<true>& words() const { return arguments_; }
    // What data() holds to the workspace (by value it is words()).
    int32_t send(void* workspace, hipStream_t stream) {
        if (by_value_) return GDN_OK;
        const size_t bytes = (size_t)ints_ * sizeof(int32_t);
        if (!slot_) return gdn::write_plan(data_, bytes, workspace, stream);
        FetchRing::Slot& s = *slot_;
        const uint32_t blocks = (uint32_t)((bytes + FETCH_PIECE - 1) / FETCH_PIECE), mark = s.mark + 1 == 0 ? 1 : s.mark + 1;
        hipLaunchKernelGGL(attn_fetch_kernel, dim3(blocks), dim3(FETCH_THREADS), 0, stream, reinterpret_cast<const u32x4*>(data_),
                           static_cast<u32x4*>(workspace), (int64_t)((bytes + 15) / 16), reinterpret_cast<uint32_t*>(s.host), mark);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_err(e);
        s.mark = mark;
        s.blocks = blocks;
        g_fetch.give_back(slot_);
        slot_ = nullptr;
        return GDN_OK;
    }

  private:
    struct Small { int32_t w[SMALL_WORDS]; };
    alignas(64) Small small_;
    alignas(64) PlanWords<true> arguments_;
    std::vector<int32_t> long_;
    int32_t* data_ = nullptr;
    int64_t ints_ = 0;
    bool by_value_ = false;
    FetchRing::Slot* slot_ = nullptr;     // this call's buffer, if it has one
};

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
    const int64_t units = ((int64_t)s->H_q + 2 * (int64_t)s->H_kv) * (s->d / 16);       // pieces of 16 elements per token
    if (units * ROPE_TOKENS > INT32_MAX) return GDN_ERR_SHAPE;
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
    rc = check_call(n_req, cu, start, pages, page_cu, page_ids, len);
    if (rc != GDN_OK) return rc;
    if (!pos) pos = start;
    for (int32_t r = 0; r < n_req; ++r)
        if (pos[r] < 0 || (int64_t)pos[r] + len[r] > INT32_MAX) return GDN_ERR_START;
    const int64_t T = cu[n_req];
    if (T == 0) return GDN_OK;
    // ---- the pages that get rows, and that nobody else in the call has them
    const int shift = shift_of(pages);
    PageSet written(pages->n_pages);
    int64_t n_written = 0;
    auto first_page = [&](int32_t r) { return start[r] >> shift; };
    auto last_page = [&](int32_t r) { return (start[r] + len[r] - 1) >> shift; };
    for (int32_t r = 0; r < n_req; ++r) {
        if (len[r] == 0) continue;
        const int32_t n = last_page(r) - first_page(r) + 1;
        if (!written.add(page_ids + page_cu[r] + first_page(r), n)) return GDN_ERR_SLOT_DUP;
        n_written += n;
    }
    bool shared = false;
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t held = (start[r] + (1 << shift) - 1) >> shift, p0 = len[r] > 0 ? first_page(r) : held;
        for (int32_t p = 0; p < p0; ++p) shared |= written.has(page_ids[page_cu[r] + p]);
    }
    if (shared) return GDN_ERR_SLOT_DUP;
    if (!q || !k || !v || !k_pool || !v_pool || !q_out) return GDN_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(q_out)) return GDN_ERR_ALIGN;
    rc = check_workspace(s, n_req, T, page_cu[n_req], workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;
    // ---- a workgroup stores its queries while others have yet to load theirs: q_out lies on q token by token, or on nothing that is read
    const int64_t size = rope->in_dtype == GDN_F32 ? 4 : 2;
    auto out_over = [&](const void* x, int64_t ld, int64_t width) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(x), out = reinterpret_cast<uintptr_t>(q_out);
        return out < lo + (uintptr_t)(((T - 1) * ld + width) * size) && lo < out + (uintptr_t)(T * wq * 2);
    };
    const bool in_place = q_out == q && size == 2 && (ldq == wq || T == 1);
    if ((!in_place && out_over(q, ldq, wq)) || out_over(k, ldk, wkv) || out_over(v, ldv, wkv)) return GDN_ERR_SLOT_HAZARD;
    Plan plan;
    rc = plan.open(4 * (int64_t)n_req + 1 + n_written, stream);
    if (rc != GDN_OK) return rc;
    int32_t* p = std::copy(cu, cu + n_req + 1, plan.data());
    p = std::copy(start, start + n_req, p);
    p = std::copy(pos, pos + n_req, p);
    int32_t *ids = p + n_req, at = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        p[r] = at - first_page(r);
        if (len[r] == 0) continue;
        const int32_t n = last_page(r) - first_page(r) + 1;
        ids = std::copy_n(page_ids + page_cu[r] + first_page(r), n, ids);
        at += n;
    }
    rc = plan.send(workspace, stream);
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
    a.tokens = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(int64_t)ROPE_TOKENS, ROPE_UNITS * ROPE_THREADS / units, (T + 255) / 256}));
    a.H_q = s->H_q; a.H_kv = s->H_kv;
    a.unit_shift = __builtin_ctz((unsigned)s->d / 16);
    a.page_shift = shift;
    a.rot = rope->rot;
    a.layout = rope->layout;
    a.amplitude = rope->amplitude;
    const dim3 grid((unsigned)((T + a.tokens - 1) / a.tokens)), block(ROPE_THREADS);
    const bool f32 = rope->in_dtype == GDN_F32;
    if (plan.by_value()) return hip_err(launch_in_place(f32 ? attn_rope_kernel<true, true> : attn_rope_kernel<false, true>, grid, block, stream, a, plan.words()));
    return hip_err(launch_in_place(f32 ? attn_rope_kernel<true, false> : attn_rope_kernel<false, false>, grid, block, stream, a, PlanWords<false>()));
}

template <bool LSE, typename Args, typename Merge>
int32_t launch_paged(const attn_shape* s, const UnitPlan& plan, const CallImage& im, const int32_t* d, bool nt, Args& a, Merge& merge, hipStream_t stream) {
    int32_t rc;
    if (im.n_narrow > 0 && (rc = launch_narrow_units<LSE>(s, nt, im, a, stream)) != GDN_OK) return rc;
    if (im.n_wide > 0 && (rc = launch_wide_units<LSE>(s, plan, im, a, stream)) != GDN_OK) return rc;
    return launch_merge<LSE, true>(s, plan, im, d, a, a.lse, a.part_le, merge, stream);
}

int32_t paged_prefill(const attn_shape* s, const void* q, const void* gate, int32_t n_req, const int32_t* cu, const int32_t* start,
                      const attn_pages* pages, const void* k_pool, const void* v_pool, const int32_t* page_cu, const int32_t* page_ids,
                      void* o, float* lse, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    int32_t rc = check_front(s, n_req, pages);
    if (rc != GDN_OK) return rc;
    if (n_req == 0) return GDN_OK;
    std::vector<int32_t> len;
    rc = check_call(n_req, cu, start, pages, page_cu, page_ids, len);
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
    build_units<true>(*s, n_req, len.data(), start, plan);
    CallImage im;
    rc = lay_out_image(s, plan, n_req, n_ids, im);
    if (rc != GDN_OK) return rc;
    Plan image;
    rc = image.open(im.ints, stream);
    if (rc != GDN_OK) return rc;
    fill_image(s, plan, n_req, cu, start, len.data(), page_cu, page_ids, n_ids, im, image.data());
    rc = image.send(workspace, stream);
    if (rc != GDN_OK) return rc;
    // by value, the arrays begin at offset 0 of the words
    const int32_t* const d = image.by_value() ? nullptr : static_cast<const int32_t*>(workspace);
    char* const parts = static_cast<char*>(workspace) + image_bytes(s, n_req, T, n_ids);
    PagedValueArgs a;
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
    if (image.by_value()) {
        CombineValueArgs merge;
        std::memcpy(a.words, image.data(), sizeof(int32_t) * (size_t)im.ints);
        std::memcpy(merge.words, image.data(), sizeof(int32_t) * (size_t)im.ints);
        return lse ? launch_paged<true>(s, plan, im, d, false, a, merge, stream) : launch_paged<false>(s, plan, im, d, false, a, merge, stream);
    }
    const bool nt = narrow_nt(s, plan, n_req, start, len.data());
    CombineArgs merge;
    PagedArgs& in_memory = a;
    return lse ? launch_paged<true>(s, plan, im, d, nt, in_memory, merge, stream) : launch_paged<false>(s, plan, im, d, nt, in_memory, merge, stream);
}

template <int D, bool BY_VALUE>
hipError_t launch_weights_d(bool few, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    if (few) return launch_in_place(attn_weights_few_kernel<D, BY_VALUE>, dim3(blocks), dim3(WGT_THREADS), stream, a, words);
    return launch_in_place(attn_weights_kernel<D, BY_VALUE>, dim3(blocks), dim3(64 * wgt_waves(D)), stream, a, words);
}
template <bool BY_VALUE>
hipError_t launch_weights(int d, bool few, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    switch (d) {
        case 64: return launch_weights_d<64>(few, a, words, blocks, stream);
        case 128: return launch_weights_d<128>(few, a, words, blocks, stream);
        default: return launch_weights_d<256>(few, a, words, blocks, stream);
    }
}
template <bool BY_VALUE>
hipError_t launch_weights_merge(int d, const WeightArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    const dim3 block((unsigned)wgt_keys(d));
    return launch_in_place(d == 256 ? attn_weights_merge_kernel<wgt_keys(256), BY_VALUE> : attn_weights_merge_kernel<wgt_keys(128), BY_VALUE>, dim3(blocks), block,
                           stream, a, words);
}

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

// The work of one attn_key_weights call: units (a tile of keys and a run of the request's query rows) of either kernel, and the tiles whose rows are cut.
struct WeightPlan {
    int64_t run = 1, most = 0;                     // row tiles per cut, and of the longest request
    int64_t n_wide = 0, n_few = 0, n_cut = 0;      // units of either kernel, cut tiles
};
// A request's tiles.
struct WeightRequest {
    bool few;
    int32_t G, start, tiles, rows, keys;
    int64_t row_tiles;
    WeightRequest(const attn_shape* s, int32_t start, int32_t len)
        : G(s->H_q / s->H_kv), start(start), keys(wgt_keys(s->d)) {
        few = len > 0 && (int64_t)len * G <= WGT_FEW;
        tiles = (int32_t)(((int64_t)start + len + keys - 1) / keys);
        rows = len * G;
        row_tiles = (rows + WGT_ROWS - 1) / WGT_ROWS;
    }
    // the first row tile that sees a key of the tile
    int64_t first_seen(int32_t tile) const { return std::max<int64_t>(0, (int64_t)tile * keys - start) * G / WGT_ROWS; }
    // tiles that every row sees a key of
    int32_t seen_by_all() const { return std::min<int32_t>(tiles, start / keys + 1); }
};

void plan_weights(const attn_shape* s, int32_t n_req, const int32_t* start, const int32_t* len, WeightPlan& out) {
    // ---- units, parts of cut tiles, cut tiles and row tiles in all if rows are cut every `run` row tiles
    int64_t work = 0;
    auto count = [&](int64_t run, int64_t& units, int64_t& parts, int64_t& cut) {
        units = parts = cut = work = 0;
        for (int32_t r = 0; r < n_req; ++r) {
            const WeightRequest q(s, start[r], len[r]);
            if (q.few) continue;
            const int64_t m = q.row_tiles;
            out.most = std::max(out.most, m);
            const RowGrid grid(run, m);
            const int64_t whole = q.seen_by_all(), cuts = m > 0 ? grid.index(m - 1) + 1 : 1;
            units += whole * cuts;
            work += whole * m;
            if (cuts > 1) { parts += whole * cuts; cut += whole; }
            for (int32_t t = (int32_t)whole; t < q.tiles; ++t) {
                const int64_t f = q.first_seen(t), p = grid.index(m - 1) - grid.index(f) + 1;
                units += p;
                work += m - f;
                if (p > 1) { parts += p; ++cut; }
            }
        }
    };
    for (int32_t r = 0; r < n_req; ++r) {
        const WeightRequest q(s, start[r], len[r]);
        if (q.few) out.n_few += q.tiles;
    }
    int64_t parts = 0;
    count(INT32_MAX, out.n_wide, parts, out.n_cut);
    out.run = std::max<int64_t>(out.most, 1);
    if (out.most <= 1) return;
    auto cost = [&](int64_t c, int64_t n) {                // units that fill every gap but half of the last short one, and no less than one unit
        const int64_t last = c < out.most ? std::max<int64_t>(1, c / 4) : c;
        const double even = (double)((work + WGT_START * n) * s->H_kv) / WGT_SLOTS + 0.5 * (double)(last + WGT_START);
        return std::max(even, (double)(c + WGT_START));
    };
    double best = cost(out.most, out.n_wide);
    for (int64_t c = out.most; c > 1;) {
        c = c > 8 ? c * 3 / 4 : c - 1;
        int64_t n, cut;
        count(c, n, parts, cut);
        if (parts * s->H_kv > WGT_PARTS) break;
        if (cost(c, n) < 0.97 * best) {
            best = cost(c, n);
            out.run = c;
            out.n_wide = n;
            out.n_cut = cut;
        }
    }
}

// The units, those of the same rows together (they read the same queries), the longest first, and the cut tiles.
void list_weights(const attn_shape* s, int32_t n_req, const int32_t* cu, const int32_t* start, const int32_t* len, const int32_t* place,
                  const WeightPlan& plan, int32_t* wide, int32_t* few, int32_t* merge) {
    struct Unit { int32_t r, kv0, lo, hi, part; };
    std::vector<Unit> list;
    list.reserve((size_t)plan.n_wide);
    std::vector<int32_t> base;
    int32_t slot = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        const WeightRequest q(s, start[r], len[r]);
        if (q.few) {
            for (int32_t t = 0; t < q.tiles; ++t, few += WGT_REC) {
                const int32_t rec[WGT_REC] = {cu[r], len[r], start[r], place[r], t * q.keys, 0, q.rows, -1};
                std::memcpy(few, rec, sizeof rec);
            }
            continue;
        }
        const int64_t m = q.row_tiles;
        if (m == 0) {
            for (int32_t t = 0; t < q.tiles; ++t) list.push_back({r, t * q.keys, 0, 0, -1});
            continue;
        }
        const RowGrid grid(plan.run, m);
        auto cut_of = [&](int32_t t) { return (int32_t)grid.index(q.first_seen(t)); };      // the first cut of rows that sees a key of tile t
        const int32_t cuts = (int32_t)grid.index(m - 1) + 1;
        base.resize(q.tiles);
        for (int32_t t = 0; t < q.tiles; ++t) {
            const int32_t parts = cuts - cut_of(t);
            base[t] = slot - cut_of(t);                  // + the cut's number: its partial sum
            if (parts <= 1) continue;
            const int32_t rec[WGT_MERGE] = {start[r] + len[r], start[r], place[r], t * q.keys, slot};
            std::memcpy(merge, rec, sizeof rec);
            merge += WGT_MERGE;
            slot += parts;
        }
        for (int32_t c = cuts - 1; c >= 0; --c) {
            const int32_t lo = (int32_t)grid.begin(c), hi = (int32_t)std::min<int64_t>(grid.begin(c + 1), m);
            for (int32_t t = 0; t < q.tiles; ++t) {
                const int32_t f = std::max(lo, (int32_t)q.first_seen(t));
                if (f >= hi) break;
                list.push_back({r, t * q.keys, f * WGT_ROWS, std::min(hi * WGT_ROWS, q.rows), cuts - cut_of(t) <= 1 ? -1 : base[t] + c});
            }
        }
    }
    if (plan.n_cut > 0) {                                 // one past the last partial sum
        const int32_t rec[WGT_MERGE] = {0, 0, 0, 0, slot};
        std::memcpy(merge, rec, sizeof rec);
    }
    // by length, in classes: a counting sort that keeps their order
    constexpr int CLASSES = 64;
    const int64_t top = std::max<int64_t>(1, std::min(plan.run, plan.most)) * WGT_ROWS;
    int32_t at[CLASSES + 1] = {0};
    auto class_of = [&](const Unit& u) { return (int)(CLASSES - 1 - (int64_t)(u.hi - u.lo) * (CLASSES - 1) / top); };
    for (const Unit& u : list) ++at[class_of(u) + 1];
    for (int i = 0; i < CLASSES; ++i) at[i + 1] += at[i];
    for (const Unit& u : list) {
        const int32_t rec[WGT_REC] = {cu[u.r], len[u.r], start[u.r], place[u.r], u.kv0, u.lo, u.hi, u.part};
        std::memcpy(wide + (size_t)at[class_of(u)]++ * WGT_REC, rec, sizeof rec);
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
    rc = check_call(n_req, cu, start, pages, page_cu, page_ids, len);
    if (rc != GDN_OK) return rc;
    const int shift = shift_of(pages);
    PageSet written(pages->n_pages);
    int64_t rows = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        const int32_t total = start[r] + len[r];
        rows += total;
        if (!written.add(page_ids + page_cu[r], ((int64_t)total + (1 << shift) - 1) >> shift)) return GDN_ERR_SLOT_DUP;
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
    WeightPlan units;
    plan_weights(s, n_req, start, len.data(), units);
    const int64_t n_wide = units.n_wide, n_few = units.n_few, n_cut = units.n_cut;
    if (std::max(n_wide, n_few) * s->H_kv > INT32_MAX) return GDN_ERR_COUNT;
    const int64_t few_at = WGT_REC * n_wide, merge_at = few_at + WGT_REC * n_few, ids_at = merge_at + (n_cut > 0 ? WGT_MERGE * (n_cut + 1) : 0);
    if ((ids_at + n_ids) * (int64_t)sizeof(int32_t) > image_bytes(s, n_req, T, n_ids)) return GDN_ERR_WORKSPACE;
    Plan plan;
    rc = plan.open(ids_at + n_ids, stream);
    if (rc != GDN_OK) return rc;
    list_weights(s, n_req, cu, start, len.data(), page_cu, units, plan.data(), plan.data() + few_at, plan.data() + merge_at);
    std::copy(page_ids, page_ids + n_ids, plan.data() + ids_at);
    rc = plan.send(workspace, stream);
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
            e = launch_weights(s->d, true, a, words, (unsigned)(n_few * s->H_kv), stream);
        }
        if (e == hipSuccess && n_wide > 0) {
            a.units = 0;
            e = launch_weights(s->d, false, a, words, (unsigned)(n_wide * s->H_kv), stream);
        }
        if (e == hipSuccess && n_cut > 0) e = launch_weights_merge(s->d, a, words, (unsigned)(n_cut * s->H_kv), stream);
        return hip_err(e);
    };
    return plan.by_value() ? launch(plan.words()) : launch(PlanWords<false>());
}

template <int D, bool BY_VALUE>
hipError_t launch_gather(const EvictArgs& a, const PlanWords<BY_VALUE>& words, unsigned blocks, hipStream_t stream) {
    return launch_in_place(attn_gather_rows_kernel<D, BY_VALUE>, dim3(blocks), dim3(GATHER_THREADS), stream, a, words);
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
    if ((int64_t)n_old + n_new > INT32_MAX) return GDN_ERR_COUNT;
    rc = check_ids(pages, page_ids, n_old);
    if (rc != GDN_OK) return rc;
    rc = check_ids(pages, new_page_ids, n_new);
    if (rc != GDN_OK) return rc;
    PageSet fresh(pages->n_pages);
    if (!fresh.add(new_page_ids, n_new)) return GDN_ERR_SLOT_DUP;
    bool hazard = false;
    for (int32_t i = 0; i < n_old; ++i) hazard |= fresh.has(page_ids[i]);
    if (hazard) return GDN_ERR_SLOT_HAZARD;
    if (total == 0) return GDN_OK;
    if (!k_pool || !v_pool || !w_pool || !index) return GDN_ERR_NULL;
    if (!aligned16(k_pool) || !aligned16(v_pool)) return GDN_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(w_pool) % 4 != 0 || reinterpret_cast<uintptr_t>(index) % 4 != 0) return GDN_ERR_ALIGN;
    rc = check_workspace(s, n_req, 0, (int64_t)n_old + n_new, workspace, workspace_bytes);
    if (rc != GDN_OK) return rc;

    const int copied = gather_rows(s->d);              // rows per workgroup of the copy
    Plan plan;
    rc = plan.open(8 * (int64_t)n_req + 2 + n_old + n_new, stream);
    if (rc != GDN_OK) return rc;
    int32_t* p = plan.data();
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
    rc = plan.send(workspace, stream);
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
        const hipError_t e = launch_in_place(attn_select_kernel<BY_VALUE>, dim3((unsigned)(n_req * s->H_kv)), dim3(SEL_THREADS), stream, a, words);
        if (e != hipSuccess) return hip_err(e);
        switch (s->d) {
            case 64: return hip_err(launch_gather<64>(a, words, (unsigned)blocks, stream));
            case 128: return hip_err(launch_gather<128>(a, words, (unsigned)blocks, stream));
            default: return hip_err(launch_gather<256>(a, words, (unsigned)blocks, stream));
        }
    };
    return plan.by_value() ? launch(plan.words()) : launch(PlanWords<false>());
}

// No exception leaves a C entry: what is thrown here is host memory that runs out, for a call of too many entries.
template <typename F>
int32_t guarded(F f) {
    try {
        return f();
    } catch (...) {
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
