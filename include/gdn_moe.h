/*
 * gdn_moe — a feed-forward block that is a mixture of experts, for one MI355X (gfx950): router, choice, the
 * chosen experts' gated products and their weighted sum.  Same library and conventions as gdn_resume.h (device
 * pointers owned by the caller, validation before anything is enqueued, negative error codes, no allocation, no
 * stream synchronisation, no atomics whose order would show in a result).
 *
 * Why it belongs to the path: in a layer group (Sec. 6, prototype wall-clock time) every replayed suffix token and every
 * decoded one passes through a feed-forward block behind each mixer; where that is a mixture of experts, a token reads k of E experts'
 * weights.  The paper does not restate the layers; what is computed is, for every token t,
 *
 *     l[e]   = sum_d x[t][d] w_router[e][d]                                   rounded once, to fp32
 *     key[e] = l[e] or sigmoid(l[e]), + choice_bias[e]                        rounded once, to fp32
 *     the k experts of the largest keys, of equal ones those of the lowest index first.  A key of -infinity is never chosen (fewer
 *     than k may be); a NaN is behind every other key that can be
 *     p[j]   = softmax over all e of l, or sigmoid(l), at the j-th choice; divided by the sum of the k with `normalise` (a
 *              sum of zero, which only logits of -infinity give, leaves zeros); * routed_scale
 *     h[j]   = p[j] * act(gate_(e_j) x[t]) * (up_(e_j) x[t])                   rounded once, to bf16
 *     y[t]   = add[t] + sum_j w_down[e_j] h[j]
 *
 * A choice whose p[j] is zero is left out of the sum, whatever its expert would give.  A token with a NaN in x has NaN weights and a NaN row y.
 *
 *   x            device, bf16, T rows of D elements at ldx elements
 *   w_router     device, router_dtype, [E][D];  choice_bias: device, fp32, [E], or NULL
 *   w_gate_up    device, bf16, [E][2 F][D]: an expert's F rows of the gate, then its F rows of up
 *   w_down       device, bf16, [E][D][F]
 *   add          device, bf16, T rows of D at ld_add elements (a shared expert's output, for one), or NULL
 *   y            device, bf16, T rows of D at ldy elements; it may be add (the same address and stride)
 *   ids          device, int32, [T][k]: the choices in the order of their keys, -1 where there is none; or NULL
 *   weights      device, fp32, [T][k]: p; or NULL
 *   workspace    device, 16-byte aligned, >= gdn_moe_workspace_bytes(shape, T); nothing in it is kept from call to call, and
 *                two calls that may run at once need one each
 *   E is 1 .. 1024, k 1 .. min(E, 16), D and F multiples of 64 up to 32768; pointers 16-byte aligned (choice_bias, ids, weights 4), ld
 *   multiples of 8 and at least D.  T = 0 is legal and does nothing.  T k is below 2^24, and x's rows (T ldx) and the experts' inner rows
 *   (T k F) span less than 2^30 elements: longer batches go in parts.
 * Arithmetic: the router's sums in fp64; bf16 products with fp32 sums in the experts; h is rounded to bf16, as the next product's
 * operand, behind its weight; the choices are added in fp32; one rounding to y.  (For few tokens a token's choices are summed as one product, for
 * more each by itself and then in the order of their keys: the same but for the order of fp32 additions.  Which it is depends on the shape and T; within a
 * call a token's row is the same bits wherever it stands.)
 * Errors: GDN_ERR_NULL, _ALIGN, _SHAPE (a size out of its range, an unknown type, activation or score, a routed_scale that is not finite, an ld
 * smaller than D), _COUNT, _WORKSPACE, _SLOT_HAZARD (y, ids, weights or the workspace share a byte with each other or an input, but for y = add).
 */
#ifndef GDN_MOE_H
#define GDN_MOE_H

#include <stdint.h>

#include "gdn_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GDN_SCORE_SOFTMAX = 0, GDN_SCORE_SIGMOID = 1 };

typedef struct gdn_moe_shape {
    int32_t E, k, D, F;
    int32_t act;                /* GDN_ACT_* of gdn_linear.h */
    int32_t score;              /* GDN_SCORE_* */
    int32_t normalise;          /* 1: the k weights are divided by their sum */
    int32_t router_dtype;       /* GDN_BF16 or GDN_F32 */
    float routed_scale;
} gdn_moe_shape;

/* Bytes of device workspace that gdn_moe needs for T tokens.  Negative on error. */
int64_t gdn_moe_workspace_bytes(const gdn_moe_shape *shape, int64_t T);

int32_t gdn_moe(const gdn_moe_shape *shape, const void *x, int64_t ldx, const void *w_router, const float *choice_bias,
                const void *w_gate_up, const void *w_down, const void *add, int64_t ld_add, void *y, int64_t ldy,
                int32_t *ids, float *weights, int64_t T, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Tuning knob, not a method step: fixes the kernels of the experts' products (0, 2, 3: tiles of 128 x 128, 256 x 256, 64 x 64, as gdn_linear_tune; 6: those
 * of few tokens where T <= 32; anything else: chosen per call, the default).  Every tile gives the same results.  Process-wide; returns the previous
 * setting (-1 = per call).
 */
int32_t gdn_moe_tune(int32_t shape);

#ifdef __cplusplus
}
#endif
#endif /* GDN_MOE_H */
