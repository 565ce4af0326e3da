/*
 * gdn_block — the residual stream between the blocks of a layer, for one MI355X (gfx950): the norm behind a
 * block, the block's gate and scale, the addition to the stream and the norm in front of the next block, in one
 * pass over the rows.  Same library and conventions as gdn_resume.h (device pointers owned by the
 * caller, validation before anything is enqueued, negative error codes, no allocation, no stream synchronisation).
 *
 * Why it belongs to the path: a layer group (Sec. 6, prototype wall-clock time) is token mixers and feed-forward blocks
 * on one stream; every replayed suffix token passes from each to the next through these rows.  The paper does not restate
 * the layers; what is computed is, for every token t,
 *
 *     s[t] = r[t] + scale * g[t] * N_post(y[t])
 *     x[t] = N_pre(s[t])
 *     N(v) = (v - m) / sqrt(mean((v - m)^2) + eps) * (w + offset) + b,    m = 0 (rms) or mean(v) (layer)
 *
 *   y      device, in_dtype, T rows of D elements at ldy elements: the block's output.  NULL: s = r (no post norm, no gate)
 *   r      device, s_dtype, rows at ldr: the stream before the block.  NULL: nothing is added
 *   s      device, s_dtype, rows at lds: the stream behind it.  NULL: not written (then x is)
 *   x      device, x_dtype, rows at ldx: the next block's input.  NULL exactly where pre is GDN_NORM_NONE
 *   gate   GDN_GATE_ELEMENT: device, in_dtype, rows at ldg; GDN_GATE_TOKEN: in_dtype, one element for a token, ldg
 *          elements apart; GDN_GATE_CHANNEL: fp32, D elements.  With gate_act = 1 its sigmoid multiplies.
 *   w, b   device, fp32, D elements.  w is needed where its norm is; b may be NULL
 *   All row strides are at least D (those of a gate per token at least 1), D and all row strides multiples of 8 (not ldg of a gate
 *   per token), pointers 16-byte aligned (a gate per token: its element).  D is 8 .. 32768.  The rows of one tensor may lie in
 *   a wider buffer.  T = 0 is legal and does nothing.
 * Arithmetic: fp32 throughout, the mean first and then the squares of what is left; x is made of the s that is held in fp32,
 * so that each output is rounded once.  A row whose mean square and eps together lie below 2^-126 (eps = 0 with a row of zeros, for
 * one) or whose squares add up past fp32's range (values of 10^17 and more) has no norm: NaN, infinities or zeros.
 * In place: s and x may each be the same rows as y, r or a gate per element (the same address, row stride and element size);
 * s and x may not share a byte, nor any output one with an input in another way.
 * Errors: GDN_ERR_NULL, _ALIGN, _SHAPE (an unknown type, norm or gate, D out of range, a row stride smaller than its row, an eps
 * that is negative or not finite, a norm or gate of a y that is not there), _COUNT (T negative or not below 2^31; a row stride above 2^40 or a tensor that spans more than 2^60
 * elements),
 * _SLOT_HAZARD (an output that overlaps an input or the other output).
 */
#ifndef GDN_BLOCK_H
#define GDN_BLOCK_H

#include <stdint.h>

#include "gdn_resume.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GDN_NORM_NONE = 0, GDN_NORM_RMS = 1, GDN_NORM_LAYER = 2 };
enum { GDN_GATE_NONE = 0, GDN_GATE_ELEMENT = 1, GDN_GATE_TOKEN = 2, GDN_GATE_CHANNEL = 3 };

typedef struct gdn_block_shape {
    int32_t D;                          /* channels */
    int32_t post, pre;                  /* GDN_NORM_* */
    int32_t in_dtype, s_dtype, x_dtype; /* GDN_F32 or GDN_BF16: y and the gate; r and s; x */
    int32_t gate, gate_act;             /* GDN_GATE_*; 0: the gate itself, 1: its sigmoid */
    float eps_post, eps_pre;
    float scale;                        /* of the block's output */
    float offset;                       /* added to both norms' weights (1 where weights are stored around zero) */
} gdn_block_shape;

int32_t gdn_block_norm(const gdn_block_shape *shape, const void *y, int64_t ldy, const void *gate, int64_t ldg,
                       const float *w_post, const float *b_post, const void *r, int64_t ldr,
                       const float *w_pre, const float *b_pre, void *s, int64_t lds, void *x, int64_t ldx,
                       int64_t T, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* GDN_BLOCK_H */
