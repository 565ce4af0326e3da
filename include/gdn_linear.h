/*
 * gdn_linear — the projections of the layers around the resumed recurrence, for one MI355X
 * (gfx950).  Same library and conventions as gdn_resume.h (device pointers owned by the caller,
 * validation before anything is enqueued, negative error codes, no allocation, no stream
 * synchronisation).
 *
 * Why it belongs to the path: the paper times a layer group of one full-attention and three
 * GatedDeltaNet layers (Sec. 6, prototype wall-clock time); in such a layer the input and output
 * projections are the largest dense products a replayed suffix token pays for.  The paper does not
 * restate them; what is computed is the affine map of any such layer,
 *
 *     y[t][n] = bias[n] + sum_k x[t][k] w[n][k] ,      t < T, n < N, k < K,
 *
 * with the weight stored [out][in] (row n of w makes output n).
 *
 *   x      device, bf16, T rows of K elements at ldx elements (ldx >= K)
 *   w      device, bf16, N rows of K elements at ldw elements (ldw >= K)
 *   bias   device, fp32, N elements, or NULL
 *   y      device, out_dtype (GDN_BF16 or GDN_F32), T rows of N elements at ldy elements (ldy >= N):
 *          y may be a column slice of a wider buffer
 *   K a multiple of 64; x, w 16-byte aligned with ldx, ldw multiples of 8; y 8-byte aligned (bf16)
 *   or 16-byte aligned (fp32) with ldy a multiple of 4.  T = 0 or N = 0 is legal and does nothing.
 * Arithmetic: bf16 products on the matrix cores, fp32 accumulation over k in the order of the
 * k index by blocks of 32; the bias is added in fp32; one rounding to out_dtype.
 * Errors: GDN_ERR_NULL, GDN_ERR_ALIGN, GDN_ERR_SHAPE (K not a multiple of 64, a leading dimension
 * smaller than its row, an unknown out_dtype), GDN_ERR_COUNT (a negative size, or a leading dimension of 4 Mi
 * elements and more: a 256-row tile is addressed with 31-bit byte offsets).
 */
#ifndef GDN_LINEAR_H
#define GDN_LINEAR_H

#include <stdint.h>

#include "gdn_resume.h"

#ifdef __cplusplus
extern "C" {
#endif

int32_t gdn_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, const float *bias,
                   void *y, int64_t ldy, int32_t out_dtype,
                   int64_t T, int32_t N, int32_t K, void *stream);

/*
 * The same map with its outputs split by column range over several destinations, in the launches of gdn_linear: segment s holds
 * outputs seg_cols[s] .. seg_cols[s + 1] - 1 and goes to seg_y[s] (T rows of that many elements at seg_ld[s]
 * elements).  This is the in-projection of a GatedDeltaNet layer as the layer's front end wants it: one weight
 * matrix [conv input | z | a | b], four separate tensors (include/gdn_layer.h); N = seg_cols[n_seg].
 *   n_seg      1 .. 8
 *   seg_cols   host, n_seg + 1, seg_cols[0] = 0, strictly increasing; inner boundaries multiples of 8
 *   seg_y      host array of n_seg device pointers (alignment as y above);  seg_ld: host, n_seg, multiples of 4
 * Everything else as gdn_linear.  Errors as gdn_linear, and GDN_ERR_COUNT for n_seg outside 1 .. 8,
 * GDN_ERR_SHAPE for seg_cols not starting at 0 or not increasing or a seg_ld below its segment's width,
 * GDN_ERR_ALIGN for an inner boundary that is no multiple of 8.
 */
int32_t gdn_linear_split(const void *x, int64_t ldx, const void *w, int64_t ldw, const float *bias,
                         int32_t n_seg, const int32_t *seg_cols, void *const *seg_y, const int64_t *seg_ld,
                         int32_t out_dtype, int64_t T, int32_t K, void *stream);

/*
 * The launches gdn_linear and gdn_linear_split make for a problem (host only; for tests and for callers that want to see
 * them): outputs 0 .. *cols - 1 in tile shape *shape and, where *cols < N, the others in a second launch in *rest_shape (shape
 * numbers as for gdn_linear_tune).  T, N, K positive (else GDN_ERR_COUNT), K a multiple of 64 (else GDN_ERR_SHAPE).
 */
int32_t gdn_linear_plan(int64_t T, int32_t N, int32_t K, int32_t *shape, int32_t *cols, int32_t *rest_shape);

/*
 * Tuning knob, not a method step: fixes the workgroup tile gdn_linear uses (0: 128 x 128; 1: 256 x 256 with four
 * waves; 2: 256 x 256 with eight waves; 3: 64 x 64; 4: 128 x 128 with three k steps in flight instead of one; 5: 128 x 160
 * like 4; anything else: chosen per call from T, N and K, the default, which
 * may also cut a large problem into two column ranges, a launch each).  Every shape computes the same
 * sums in the same order, so the results do not depend on it.  Process-wide; returns the previous setting (-1 = per
 * call).
 */
int32_t gdn_linear_tune(int32_t shape);

/*
 * The map with an epilogue: activation, a second product as the gate's counterpart, a factor and a residual, as the two products of a
 * feed-forward block want them,
 *
 *     z[t][n] = bias[n] + sum_k x[t][k] w[n][k]
 *     a       = act(z)                                                     without w_up
 *     a       = act(z) * (bias_up[n] + sum_k x[t][k] w_up[n][k])           with it (w is the gate's weight)
 *     y[t][n] = scale * a + residual[t][n]
 *
 *   w_up      device, bf16, N rows of K at ldw_up elements, or NULL;  bias_up: device, fp32, N, or NULL (also without w_up)
 *   residual  device, res_dtype, T rows of N elements at ldr elements (alignment as y of that type), or NULL; it may be y itself (the
 *             same address, ldr = ldy, res_dtype = out_dtype).  Otherwise y shares no byte with x, w, w_up, a bias or the residual
 * Everything else as gdn_linear.  Arithmetic: fp32 sums of the bf16 products; act, factor and residual in fp32; one rounding to out_dtype.
 * The activations are off by a few units of 2^-23 of their value, and where that is small because z is far below zero by as many as their exponential's argument
 * beside it, twice at most (|z|; GELU: z^2 / 2; by tanh: 1.6 (|z| + 0.045 |z|^3)).
 * For at most 1024 rows the sum over k may be taken in four parts that are added in order (whether and which: by T, N and K alone), else it is
 * gdn_linear's.  Errors as gdn_linear, and GDN_ERR_NULL without an epilogue, GDN_ERR_SHAPE for an unknown activation or res_dtype, a bias_up
 * without w_up, ldr < N or ldw_up < K, GDN_ERR_COUNT for N from 2^24 on or a y or residual with a row stride above 2^30 or a
 * span of more than 2^60 elements, GDN_ERR_SLOT_HAZARD where y shares bytes as said.
 */
enum { GDN_ACT_NONE = 0, GDN_ACT_SILU = 1, GDN_ACT_GELU = 2, GDN_ACT_GELU_TANH = 3, GDN_ACT_RELU = 4, GDN_ACT_RELU2 = 5, GDN_ACT_SIGMOID = 6 };

typedef struct gdn_linear_epilogue {
    int32_t act;               /* GDN_ACT_*; GELU by the error function or by tanh; RELU2: the square of RELU */
    int32_t res_dtype;         /* GDN_BF16 or GDN_F32 (of a residual that is there) */
    float scale;
    const void *w_up;
    int64_t ldw_up;
    const float *bias_up;
    const void *residual;
    int64_t ldr;
} gdn_linear_epilogue;

int32_t gdn_linear_act(const void *x, int64_t ldx, const void *w, int64_t ldw, const float *bias,
                       const gdn_linear_epilogue *epilogue, void *y, int64_t ldy, int32_t out_dtype,
                       int64_t T, int32_t N, int32_t K, void *stream);

/* gdn_linear_plan of gdn_linear_act; gated: 1 with a w_up.  Shapes 6 .. 11: the kernels of few rows, for T <= 1024. */
int32_t gdn_linear_act_plan(int64_t T, int32_t N, int32_t K, int32_t gated, int32_t *shape, int32_t *cols, int32_t *rest_shape);

/*
 * gdn_linear_tune of gdn_linear_act: 0 .. 5 (1 is 2, and with a w_up 5 is 0); 6 .. 11 the kernels of few rows where T <= 1024, workgroups of
 * 16 rows of x with 8, 16 or 32 of w, then of 32 with each (8 is 16 with a w_up); anything else: chosen per call.
 */
int32_t gdn_linear_act_tune(int32_t shape);

#ifdef __cplusplus
}
#endif
#endif /* GDN_LINEAR_H */
