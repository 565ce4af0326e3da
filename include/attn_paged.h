/*
 * attn_paged — an attention layer's keys and values in pages, for one MI355X (gfx950): rotary positions with the
 * append, attention of a chunk of new tokens, the attention weight every cached row gathers, and eviction by that
 * weight.  Same library and conventions as attn_resume.h (host / device pointers named per argument, validation
 * before anything is enqueued, negative error codes, no device allocation, no stream synchronisation: a call whose index arrays need a
 * pinned staging buffer, more than 1792 words of page ids and plan, waits for one of eight for 2 ms at most).  Under graph capture such
 * a call is refused with the capture's error; a replay of a smaller one repeats its arrays.
 *
 * The cache.  A pool of n_pages pages per tensor; page p is at pool + p * page_stride (elements) and holds
 * page_rows rows of every key/value head, [H_kv][page_rows][d]: keys in bf16, values in fp16 (as in attn_resume.h: the
 * append widens bf16 to fp16, exact for magnitudes in [2^-14, 65504], rounded to a multiple of 2^-24 below, infinite
 * above).  Row j of request r lies in row j % page_rows of page page_ids[page_cu[r] + j / page_rows]: page_cu (n_req + 1
 * ints, from 0) and page_ids are host arrays.  Requests may share pages (a common cached prefix), wherever the call
 * only reads them.  What a page holds behind its request's last row is never used, whatever it is.
 *
 *   request r holds start[r] = c rows and brings n = cu_seqlens[r+1] - cu_seqlens[r] new tokens, of which token i
 *   (0-based) becomes row c + i and sees the rows 0 .. c + i.
 *
 * A row's place is not its position: rotary positions are an argument of their own, and after an eviction a request
 * goes on with fewer rows and the same positions.
 */
#ifndef ATTN_PAGED_H
#define ATTN_PAGED_H

#include <stdint.h>

#include "attn_resume.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The geometry of a pool of pages (of keys and of values alike). */
typedef struct attn_pages {
    int64_t page_stride;  /* elements from one page to the next: a multiple of 8, at least H_kv * page_rows * d */
    int32_t n_pages;
    int32_t page_rows;    /* rows per page: a power of two, 16 .. 256 (and H_kv * page_rows * d * 2 < 2^31) */
} attn_pages;

/* Rotary positions: the first `rot` elements of a head turn in pairs, the others stay as they are. */
typedef struct attn_rope {
    int32_t rot;           /* a multiple of 16, 0 .. d */
    int32_t layout;        /* 0: the pairs are (p, p + rot/2); 1: (2p, 2p + 1) */
    int32_t in_dtype;      /* GDN_BF16 or GDN_F32: type of q, k and v as they come */
    float amplitude;       /* multiplies cosine and sine; finite */
    const double *freq;    /* host: rot / 2 angles per position (radians, finite), pair p's turning by position * freq[p] */
} attn_rope;

/* How attn_rope_freqs stretches the positions of a model to longer contexts. */
enum {
    ATTN_ROPE_PLAIN = 0,   /* base^(-2p/rot) */
    ATTN_ROPE_LINEAR = 1,  /* that over `factor`: positions are interpolated */
    ATTN_ROPE_BASE = 2,    /* base * factor^(rot/(rot-2)) in place of base: the fastest pair stays, the slowest is slowed by factor */
    ATTN_ROPE_RAMP = 3     /* pairs of more than `fast` turns in `context` positions stay, those of fewer than `slow` are slowed by
                              factor, a linear ramp over p between the two (each end rounded outwards); amplitude 0.1 ln(factor) + 1 */
};

/*
 * Host only: the rot / 2 frequencies (radians per position, fp64) of a kind of scaling, and its amplitude.
 *   base > 1, factor >= 1 finite;  ATTN_ROPE_RAMP: context > 0, fast > slow > 0
 * Errors: GDN_ERR_NULL, _SHAPE.
 */
int32_t attn_rope_freqs(int32_t rot, double base, int32_t kind, double factor, double context, double fast, double slow,
                        double *freq, double *amplitude);

/*
 * Bytes of device workspace that each of the calls below needs, for n_req requests of total_tokens new tokens
 * (attn_evict: 0) and n_page_ids listed pages (attn_evict: old and new ones).  Negative on error.
 */
int64_t attn_paged_workspace_bytes(const attn_shape *shape, int32_t n_req, int64_t total_tokens, int64_t n_page_ids);

/*
 * Rotates the queries and keys of the new tokens and appends keys and values to the pages:
 *   phi = (pos[r] + i) * freq[p];   (x, y) -> amplitude * (x cos phi - y sin phi, y cos phi + x sin phi)
 * Angles are reduced in 64 bits (2^-64 turns per position), cosine, sine and the rotation are fp32; q and k are rounded
 * to bf16 once.  One launch behind the upload of the index arrays.
 *   q, k, v      device, in_dtype, [T][H_q][d] and [T][H_kv][d], tokens ldq, ldk, ldv elements apart (16-byte multiples:
 *                they may be column ranges of one projection's output)
 *   pos          host, n_req: the position of each request's first new token, >= 0; NULL: start
 *   q_out        device, bf16, [T][H_q][d]; may be q itself where q is bf16 and ldq = H_q * d (or T is 1), and lies over no other
 *                part of q, k or v
 *   k_pool, v_pool  device; the pages that get rows belong to one request alone and are listed once in the call
 *   shape        H_q, H_kv and d are used
 * Errors: GDN_ERR_NULL, _ALIGN, _SHAPE, _SEQLENS, _START (a negative start or position, positions beyond 2^31 - 1, or
 * too few pages for the rows), _COUNT, _SLOT_RANGE (a page id outside the pool), _SLOT_DUP, _SLOT_HAZARD (q_out over what is read),
 * _WORKSPACE.
 */
int32_t attn_rope_append(const attn_shape *shape, const attn_rope *rope, const void *q, int64_t ldq, const void *k, int64_t ldk,
                         const void *v, int64_t ldv, int32_t n_req, const int32_t *cu_seqlens, const int32_t *pos,
                         const int32_t *start, const attn_pages *pages, void *k_pool, void *v_pool, const int32_t *page_cu,
                         const int32_t *page_ids, void *q_out, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Causal softmax attention of the new tokens over their requests' rows, the new ones among them (they are in the pages
 * already, by attn_rope_append):
 *   o_t[h] = sum_{j <= c+t} softmax_j(scale * q_t[h] . k_j[g]) v_j[g],  g = h / (H_q / H_kv);  times sigmoid(gate_t[h])
 *   lse_t[h] = ln sum_{j <= c+t} exp(scale * q_t[h] . k_j[g])
 * Precision, launches, and how walks are packed are those of attn_suffix_prefill, the tuning knobs too; small calls cut their
 * walks from 512 keys on (256 at d = 256), and what is not cut has that call's bits.  lse comes from a sum of the weights before
 * their rounding.  What a later token's key and value rows hold, infinities and NaN
 * included, does not reach the rows before it.
 *   q            device, bf16, [T][H_q][d];  out_gate: device, bf16, [T][H_q][d] or NULL
 *   o            device, o_dtype, [T][H_q][d];  lse: device, fp32, [T][H_q] or NULL
 * Errors: as above (pages may be shared: no _SLOT_DUP).
 */
int32_t attn_paged_prefill(const attn_shape *shape, const void *q, const void *out_gate, int32_t n_req, const int32_t *cu_seqlens,
                           const int32_t *start, const attn_pages *pages, const void *k_pool, const void *v_pool,
                           const int32_t *page_cu, const int32_t *page_ids, void *o, float *lse, void *workspace,
                           int64_t workspace_bytes, void *stream);

/*
 * The attention weight that every cached row gathers from the new tokens, summed over the query heads of its group:
 *   w_out_j[g] = decay * w_in_j[g] + sum_{t: c+t >= j} sum_{h of g} exp(scale * q_t[h] . k_j[g] - lse_t[h])
 * for the rows j < c + n of every request; the new rows (j >= c) have no w_in.  All in fp32, the sums in an order that
 * the call's sizes fix.
 *   q, lse       as attn_paged_prefill took and left them
 *   w_in, w_out  device, fp32, pools of pages [H_kv][page_rows] w_stride floats apart, under the page ids of the keys; w_in may
 *                be w_out, or NULL (nothing gathered yet).  Every page is listed once in the call.
 *   decay        finite
 * Errors: as above.
 */
int32_t attn_key_weights(const attn_shape *shape, const void *q, const float *lse, int32_t n_req, const int32_t *cu_seqlens,
                         const int32_t *start, const attn_pages *pages, const void *k_pool, const int32_t *page_cu,
                         const int32_t *page_ids, float decay, const float *w_in, float *w_out, int64_t w_stride, void *workspace,
                         int64_t workspace_bytes, void *stream);

/*
 * Eviction: of the rows[r] rows of request r each key/value head keeps min(keep[r], rows[r]) = m: the first first[r], the
 * last recent[r], and of those between the m - first[r] - recent[r] of the largest weight (equal weights: the lower row
 * first; a weight that is not a number counts below every number).  The kept rows of k, v and w are
 * copied, in their order, to rows 0 .. m-1 of the request's new pages; the old pages stay as they are.
 *   rows, keep, first, recent   host, n_req, >= 0;  first + recent <= m
 *   new_page_cu, new_page_ids   host: the new pages, each listed once, none of them an old page of the call
 *   index        device, int32: row numbers, those of request r and head g at H_kv * (m of the requests before r) + g * m
 * Errors: as above; GDN_ERR_START where first + recent exceed m or pages are too few, _SLOT_DUP, _SLOT_HAZARD (a new page among
 * the old ones).
 */
int32_t attn_evict(const attn_shape *shape, int32_t n_req, const int32_t *rows, const int32_t *keep, const int32_t *first,
                   const int32_t *recent, const attn_pages *pages, void *k_pool, void *v_pool, float *w_pool, int64_t w_stride,
                   const int32_t *page_cu, const int32_t *page_ids, const int32_t *new_page_cu, const int32_t *new_page_ids,
                   int32_t *index, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_PAGED_H */
