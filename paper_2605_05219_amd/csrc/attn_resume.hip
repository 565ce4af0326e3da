// attn_resume: host side of the attention layers' part of a cache hit (see include/attn_resume.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "attn_launch.h"

namespace attn {

// Appends the suffix's key and value rows to the cache rows start .. start+n-1 of each request's
// slot: one 16-byte chunk of k and of v per thread, the values widened from bf16 to fp16.
__global__ void __launch_bounds__(APPEND_THREADS) attn_append_kernel(AppendArgs a) {
    const int64_t id = (int64_t)blockIdx.x * APPEND_THREADS + threadIdx.x;
    if (id >= a.n_chunks) return;
    const int32_t t = (int32_t)(id / a.row_chunks);
    const int32_t c = (int32_t)(id - (int64_t)t * a.row_chunks);
    int lo = 0, hi = a.n_req;                       // request with cu[r] <= t < cu[r+1]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] <= t) lo = mid; else hi = mid;
    }
    const int r = lo;
    if (a.start[r] < 0) return;
    const int64_t row = (int64_t)a.start[r] + (t - a.cu[r]);
    const int64_t dst = (int64_t)a.slot[r] * a.slot_stride + (row * a.row_chunks + c) * 8;
    const int64_t src = ((int64_t)t * a.row_chunks + c) * 8;
    append_chunk(a.k_new + src, a.v_new + src, a.k_cache + dst, a.v_cache + dst);
}

namespace {

// geometry of a pool of sequence slots
int32_t check_pool(const attn_shape* s, int64_t slot_stride, int32_t n_slots, int32_t cap) {
    if (n_slots < 0 || cap < 0) return GDN_ERR_COUNT;
    if (slot_stride < 0 || slot_stride % 8 != 0) return GDN_ERR_ALIGN;
    if (slot_stride < (int64_t)cap * s->H_kv * s->d) return GDN_ERR_SHAPE;   // slots would overlap
    // a slot is addressed with 32-bit byte offsets, which may run up to two key tiles past its last row
    if (((int64_t)cap + 128) * s->H_kv * s->d * 2 > INT32_MAX) return GDN_ERR_SHAPE;
    return GDN_OK;
}

int32_t check_slots(const int32_t* ids, int32_t n, int32_t n_slots, bool skip_empty, const int32_t* len) {
    std::vector<int32_t> seen;
    seen.reserve(n);
    for (int32_t r = 0; r < n; ++r) {
        if (ids[r] < 0 || ids[r] >= n_slots) return GDN_ERR_SLOT_RANGE;
        if (skip_empty && len[r] == 0) continue;
        seen.push_back(ids[r]);
    }
    std::sort(seen.begin(), seen.end());
    if (std::adjacent_find(seen.begin(), seen.end()) != seen.end()) return GDN_ERR_SLOT_DUP;
    return GDN_OK;
}

// The requests of attn_plan and attn_plan_heads checked, and their suffix lengths.
int32_t plan_lengths(int32_t n_req, const int32_t* cu_seqlens, const int32_t* start_pos, std::vector<int32_t>& len) {
    len.resize(n_req);
    if (!cu_seqlens || !start_pos) return GDN_ERR_NULL;
    if (cu_seqlens[0] != 0) return GDN_ERR_SEQLENS;
    for (int32_t r = 0; r < n_req; ++r) {
        if (cu_seqlens[r + 1] < cu_seqlens[r]) return GDN_ERR_SEQLENS;
        len[r] = cu_seqlens[r + 1] - cu_seqlens[r];
        if (start_pos[r] < 0 || (int64_t)start_pos[r] + len[r] > INT32_MAX - 256) return GDN_ERR_START;
    }
    return GDN_OK;
}

}  // namespace
}  // namespace attn

using namespace attn;

extern "C" {

int64_t attn_workspace_bytes(const attn_shape* s, int32_t n_req, int64_t total_tokens) {
    const int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0 || total_tokens < 0) return GDN_ERR_COUNT;
    return plan_bytes(n_req, total_tokens, s->H_q / s->H_kv) + part_ml_bytes() + part_o_bytes(s->d);
}

// shared by attn_kv_restore and attn_kv_spill: rows [0, n_rows[r]) of one pool's slot to the other's
static int32_t kv_tier_copy(const attn_shape* s, int32_t n_req, const int32_t* n_rows, void* host_k, void* host_v,
                            int64_t host_slot_stride, int32_t n_host_slots, const int32_t* host_slot, void* k_cache, void* v_cache,
                            int64_t slot_stride, int32_t n_slots, int32_t cap, const int32_t* seq_slot, bool to_device,
                            hipStream_t stream) {
    int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0 || n_host_slots < 0) return GDN_ERR_COUNT;
    rc = check_pool(s, slot_stride, n_slots, cap);
    if (rc != GDN_OK) return rc;
    rc = check_pool(s, host_slot_stride, n_host_slots, cap);
    if (rc != GDN_OK) return rc;
    if (n_req == 0) return GDN_OK;
    if (!n_rows || !host_slot || !seq_slot) return GDN_ERR_NULL;
    int64_t total = 0;
    for (int32_t r = 0; r < n_req; ++r) {
        if (n_rows[r] < 0 || n_rows[r] > cap) return GDN_ERR_START;
        total += n_rows[r];
    }
    // the source slots only have to exist; the destination slots must also differ
    for (int32_t r = 0; r < n_req; ++r) {
        if (host_slot[r] < 0 || host_slot[r] >= n_host_slots) return GDN_ERR_SLOT_RANGE;
        if (seq_slot[r] < 0 || seq_slot[r] >= n_slots) return GDN_ERR_SLOT_RANGE;
    }
    rc = to_device ? check_slots(seq_slot, n_req, n_slots, false, nullptr) : check_slots(host_slot, n_req, n_host_slots, false, nullptr);
    if (rc != GDN_OK) return rc;
    if (total == 0) return GDN_OK;
    if (!host_k || !host_v || !k_cache || !v_cache) return GDN_ERR_NULL;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return GDN_ERR_ALIGN;
    const int64_t row = (int64_t)s->H_kv * s->d;
    for (int32_t r = 0; r < n_req; ++r) {
        if (n_rows[r] == 0) continue;
        const size_t bytes = (size_t)n_rows[r] * row * sizeof(uint16_t);
        const int64_t ho = (int64_t)host_slot[r] * host_slot_stride, dv = (int64_t)seq_slot[r] * slot_stride;
        uint16_t* const hk = static_cast<uint16_t*>(host_k) + ho;
        uint16_t* const hv = static_cast<uint16_t*>(host_v) + ho;
        uint16_t* const dk = static_cast<uint16_t*>(k_cache) + dv;
        uint16_t* const dvp = static_cast<uint16_t*>(v_cache) + dv;
        hipError_t e = to_device ? hipMemcpyAsync(dk, hk, bytes, hipMemcpyHostToDevice, stream)
                                 : hipMemcpyAsync(hk, dk, bytes, hipMemcpyDeviceToHost, stream);
        if (e != hipSuccess) return hip_err(e);
        e = to_device ? hipMemcpyAsync(dvp, hv, bytes, hipMemcpyHostToDevice, stream)
                      : hipMemcpyAsync(hv, dvp, bytes, hipMemcpyDeviceToHost, stream);
        if (e != hipSuccess) return hip_err(e);
    }
    return GDN_OK;
}

int32_t attn_kv_restore(const attn_shape* s, int32_t n_req, const int32_t* prefix_len, const void* host_k, const void* host_v,
                        int64_t host_slot_stride, int32_t n_host_slots, const int32_t* host_slot, void* k_cache, void* v_cache,
                        int64_t slot_stride, int32_t n_slots, int32_t cap, const int32_t* seq_slot, void* stream) {
    return kv_tier_copy(s, n_req, prefix_len, const_cast<void*>(host_k), const_cast<void*>(host_v), host_slot_stride, n_host_slots,
                        host_slot, k_cache, v_cache, slot_stride, n_slots, cap, seq_slot, true, static_cast<hipStream_t>(stream));
}

int32_t attn_kv_spill(const attn_shape* s, int32_t n_req, const int32_t* n_rows, void* host_k, void* host_v,
                      int64_t host_slot_stride, int32_t n_host_slots, const int32_t* host_slot, const void* k_cache,
                      const void* v_cache, int64_t slot_stride, int32_t n_slots, int32_t cap, const int32_t* seq_slot, void* stream) {
    return kv_tier_copy(s, n_req, n_rows, host_k, host_v, host_slot_stride, n_host_slots, host_slot, const_cast<void*>(k_cache),
                        const_cast<void*>(v_cache), slot_stride, n_slots, cap, seq_slot, false, static_cast<hipStream_t>(stream));
}

int32_t attn_plan(const attn_shape* s, int32_t n_req, const int32_t* cu_seqlens, const int32_t* start_pos, int32_t capacity,
                  int32_t* unit_req, int32_t* unit_tile, int32_t* unit_t0, int32_t* unit_t1, int32_t* unit_part,
                  int32_t* n_units, int32_t* heads_per_row_group, int32_t* key_tile_rows) {
    int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0 || capacity < 0) return GDN_ERR_COUNT;
    if (!n_units || !heads_per_row_group || !key_tile_rows) return GDN_ERR_NULL;
    *n_units = 0;
    *heads_per_row_group = 1;
    *key_tile_rows = att_kt(s->d);
    if (n_req == 0) return GDN_OK;
    std::vector<int32_t> len;
    rc = plan_lengths(n_req, cu_seqlens, start_pos, len);
    if (rc != GDN_OK) return rc;
    UnitPlan plan;
    build_units<false>(*s, n_req, len.data(), start_pos, plan);
    *n_units = (int32_t)plan.units.size();
    *heads_per_row_group = plan.apart && plan.n_units[0] == 0 ? s->H_q / s->H_kv : plan.pack;
    if ((int64_t)plan.units.size() > capacity) return GDN_ERR_COUNT;
    if (!plan.units.empty() && (!unit_req || !unit_tile || !unit_t0 || !unit_t1 || !unit_part)) return GDN_ERR_NULL;
    for (size_t i = 0; i < plan.units.size(); ++i) {
        unit_req[i] = plan.units[i].req;
        unit_tile[i] = plan.units[i].tile;
        unit_t0[i] = plan.units[i].t0;
        unit_t1[i] = plan.units[i].t1;
        unit_part[i] = plan.units[i].part < 0 ? -1 : plan.units[i].part + (plan.units[i].few ? plan.n_slots[0] : 0);
    }
    return GDN_OK;
}

int32_t attn_plan_heads(const attn_shape* s, int32_t n_req, const int32_t* cu_seqlens, const int32_t* start_pos) {
    int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0) return GDN_ERR_COUNT;
    if (n_req == 0) return 1;
    std::vector<int32_t> len;
    rc = plan_lengths(n_req, cu_seqlens, start_pos, len);
    if (rc != GDN_OK) return rc;
    UnitPlan plan;
    build_units<false>(*s, n_req, len.data(), start_pos, plan);
    return heads_per_workgroup(*s, plan);
}

int32_t attn_suffix_prefill(const attn_shape* s, const void* q, const void* k_new, const void* v_new, const void* out_gate,
                            int32_t n_req, const int32_t* cu_seqlens, const int32_t* start_pos, void* k_cache, void* v_cache,
                            int64_t slot_stride, int32_t n_slots, int32_t cap, const int32_t* seq_slot, void* o, void* workspace,
                            int64_t workspace_bytes, void* stream_v) {
    hipStream_t stream = static_cast<hipStream_t>(stream_v);
    int32_t rc = check_shape(s);
    if (rc != GDN_OK) return rc;
    if (n_req < 0) return GDN_ERR_COUNT;
    rc = check_pool(s, slot_stride, n_slots, cap);
    if (rc != GDN_OK) return rc;
    if (n_req == 0) return GDN_OK;
    if (!cu_seqlens || !start_pos || !seq_slot) return GDN_ERR_NULL;
    if (cu_seqlens[0] != 0) return GDN_ERR_SEQLENS;
    std::vector<int32_t> len(n_req);
    for (int32_t r = 0; r < n_req; ++r) {
        if (cu_seqlens[r + 1] < cu_seqlens[r]) return GDN_ERR_SEQLENS;
        len[r] = cu_seqlens[r + 1] - cu_seqlens[r];
        if (start_pos[r] < 0 || (int64_t)start_pos[r] + len[r] > cap) return GDN_ERR_START;
    }
    rc = check_slots(seq_slot, n_req, n_slots, true, len.data());
    if (rc != GDN_OK) return rc;
    const int64_t T = cu_seqlens[n_req];
    if (T == 0) return GDN_OK;
    if (!q || !k_new || !v_new || !k_cache || !v_cache || !o) return GDN_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o) ||
        !aligned16(out_gate))
        return GDN_ERR_ALIGN;
    if (!workspace || !aligned16(workspace) || workspace_bytes < attn_workspace_bytes(s, n_req, T)) return GDN_ERR_WORKSPACE;

    UnitPlan plan;
    build_units<false>(*s, n_req, len.data(), start_pos, plan);
    CallImage im;
    rc = lay_out_image(s, plan, n_req, 0, im);
    if (rc != GDN_OK) return rc;
    std::vector<int32_t> img((size_t)im.ints, 0);
    fill_image(s, plan, n_req, cu_seqlens, start_pos, len.data(), seq_slot, nullptr, 0, im, img.data());
    rc = gdn::upload_plan(img.data(), img.size() * sizeof(int32_t), workspace, stream);
    if (rc != GDN_OK) return rc;
    const int32_t* d = static_cast<const int32_t*>(workspace);

    SlotNarrowArgs a;
    a.q = static_cast<const uint16_t*>(q);
    a.gate = static_cast<const uint16_t*>(out_gate);
    a.k_cache = static_cast<const uint16_t*>(k_cache);
    a.v_cache = static_cast<const uint16_t*>(v_cache);
    a.o = o;
    a.slot_stride = slot_stride;
    image_args(s, plan, n_req, im, d, static_cast<char*>(workspace) + plan_bytes(n_req, T, s->H_q / s->H_kv), a);
    AppendArgs& ap = a.ap;
    ap.k_new = static_cast<const uint16_t*>(k_new);
    ap.v_new = static_cast<const uint16_t*>(v_new);
    ap.k_cache = static_cast<uint16_t*>(k_cache);
    ap.v_cache = static_cast<uint16_t*>(v_cache);
    ap.cu = a.cu;
    ap.start = a.start;
    ap.slot = a.slot;
    ap.slot_stride = slot_stride;
    ap.row_chunks = s->H_kv * s->d / 8;
    ap.n_chunks = T * ap.row_chunks;
    ap.n_req = n_req;
    const int64_t ablocks = (ap.n_chunks + APPEND_THREADS - 1) / APPEND_THREADS;
    if (ablocks > INT32_MAX) return GDN_ERR_COUNT;
    if (im.n_wide > 0) {                       // (the few-rows kernel appends its own rows)
        hipLaunchKernelGGL(attn_append_kernel, dim3((unsigned)ablocks), dim3(APPEND_THREADS), 0, stream, ap);
        rc = hip_err(hipGetLastError());
        if (rc != GDN_OK) return rc;
    }
    if (im.n_narrow > 0) {
        rc = launch_narrow_units<false>(s, narrow_nt(s, plan, n_req, start_pos, len.data()), im, a, stream);
        if (rc != GDN_OK) return rc;
    }
    if (im.n_wide > 0) {
        rc = launch_wide_units<false>(s, plan, im, static_cast<AttnArgs&>(a), stream);
        if (rc != GDN_OK) return rc;
    }
    CombineArgs ca;
    return launch_merge<false, false>(s, plan, im, d, a, nullptr, nullptr, ca, stream);
}

int32_t attn_tune_split(int32_t allow) { return g_allow_split.exchange(allow != 0); }

int32_t attn_tune_pack(int32_t allow) { return g_allow_pack.exchange(allow != 0); }

int32_t attn_tune_pairs(int32_t mode) { return g_pairs.exchange(mode == 0 || mode == 2 ? mode : 1); }

}  // extern "C"
