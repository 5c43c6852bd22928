/*
 * fp8_norm.h -- the norm between two FP8 linears of fp8lin.h, forward and backward (the conventions stated there hold here
 * too: status codes, device pointers, streams, no allocation, no synchronisation, argument errors returned before anything
 * is launched).
 *
 * The paper quantises the linears only; in a GPT or Llama decoder each of them reads the output of a layer norm (or of its
 * root-mean-square form).  Section 3 names the cost that FP8-AMAX adds there: a second round trip to memory, for the amax
 * and then for the bytes.  Here the norm takes the amax while it normalises and writes the bytes that the linear reads, so
 * that its 16-bit output need not exist.
 *
 *     h    = x + residual                      rounded to the tensors' type (x itself where there is no residual)
 *     mean = sum_j h_j / cols (0 for FP8_NORM_RMS),  rstd = 1 / sqrt(sum_j (h_j - mean)^2 / cols + eps)
 *     y    = (h - mean) * rstd * weight + bias_vec      in FP32, rounded once to the tensors' type
 *     y8   = RNE_E4(y * 2^(bias + delta)), saturating, exactly what fp8_cast_e4 makes of y
 * Sums are FP32; the variance is taken from deviations from the mean.  A row whose sum or squares FP32 does not hold is summed
 * again, its deviations times 2^-96 or 2^96.  A row with a NaN gives NaN, the statistics too; so does one with an infinity in a
 * layer norm.  FP8_NORM_RMS has rstd = 1 / infinity = 0 there: y is bias_vec, NaN where the infinity is.
 */
#ifndef FP8_NORM_H
#define FP8_NORM_H

#include "fp8lin.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FP8_NORM_LAYER = 0, FP8_NORM_RMS = 1 } fp8_norm_kind_t;

/* Tensors [rows][cols] of type dt, rows ld_* elements apart; vectors of cols elements of type w_dt (dt or FP8_F32).
 *   x            in
 *   residual     NULL, or in
 *   weight       NULL (ones), or in;   bias_vec   NULL (zeros), or in
 *   h            NULL, or out: x + residual.  May be x or residual itself (rows as far apart); no other output
 *                may overlap an input.
 *   y            NULL, or out
 *   d_mean       NULL, or out float [rows] (zeros for FP8_NORM_RMS);   d_rstd   NULL, or out float [rows]
 *   y8           NULL, or out, [rows][cols] contiguous E4 bytes
 *   d_bias_in    NULL, or the bias to cast under (FP8-CSCALE, amax history): one pass.  NULL: the bias of Eq. 3 for the
 *                amax of y, minus margin: d_bias_out, d_rstd and (layer norm) d_mean are required with y8 then.
 *   d_amax       NULL, or out: amax of y;   d_bias_out   NULL, or out: the bias of Eq. 3 (E4) for it, minus margin
 *   FP8_FLAG_NONFINITE_AMAX, FP8_FLAG_ZERO_AMAX and FP8_FLAG_SATURATED are raised as fp8_cast_e4 raises them.
 * At least one of h, y, d_mean, d_rstd, y8, d_amax, d_bias_out.  eps >= 0 and finite.  cols up to 2^30.  Pointers and
 * distances need the alignment of an element.  Rows of up to 16384 columns that are 16-byte aligned in all tensors (y8: 8-byte),
 * with cols a multiple of 8 (4 in FP32), take the fast kernels; FP32 rows with a residual up to 14272 columns.  The other kernels
 * go element by element.  Of the fast ones' statistics and output a row has the same bits in every call. */
typedef struct {
    const void *x, *residual, *weight, *bias_vec;
    void *h, *y;
    float *d_mean, *d_rstd;
    uint8_t *y8;
    const int32_t *d_bias_in;
    float *d_amax;
    int32_t *d_bias_out;
    int64_t rows, cols, ld_x, ld_residual, ld_h, ld_y;
    int32_t kind, dt, w_dt, conv, margin; /* fp8_norm_kind_t, fp8_dtype_t, fp8_dtype_t, fp8_conv_t */
    float eps;
} fp8_norm_fwd_t;
FP8_API fp8_status_t fp8_norm_fwd(fp8_ctx *ctx, const fp8_norm_fwd_t *args, void *stream);

/* The backward pass, from the sum h and the statistics that the forward pass left.  With xh = (h - mean) * rstd and
 * g = dy * weight:
 *     dx = rstd * (g - avg_j g - xh * avg_j (g xh)) + dh       (without avg_j g for FP8_NORM_RMS)
 *     dw = sum over rows of dy * xh,   db = sum over rows of dy
 * in FP32, rounded once.  dx is the gradient of x and of the residual alike.
 *   dy, h        in, [rows][cols] of dt;   dh   NULL, or in: the gradient that reaches h beside the norm
 *   weight       NULL (ones), or in, of w_dt
 *   d_mean       in, float [rows] (not read for FP8_NORM_RMS, may be NULL);   d_rstd   in, float [rows]
 *   dx           NULL, or out, of dt.  May be dy or dh itself (rows as far apart).
 *   dw, db       NULL, or out, [cols] of w_dt.  Sums over rows are taken in an order that depends on the sizes, the type, whether
 *                there is dh and which kernel the alignment allows, not on the order in which blocks arrive: a call made again
 *                gives the same bits.
 *   d_amax       NULL, or out: amax of dx (its E5 cast in the linear below needs no pass of its own; needs dx)
 * At least one of dx, dw, db.  dw and db use the context's workspace: calls that share one fp8_ctx must not overlap on the
 * device, like decode-size matmuls.  cols up to 2^22 where dw or db is asked for.  Fast kernels as above, FP32 rows up to 14272
 * columns, 9512 with dh. */
typedef struct {
    const void *dy, *h, *dh, *weight;
    const float *d_mean, *d_rstd;
    void *dx, *dw, *db;
    float *d_amax;
    int64_t rows, cols, ld_dy, ld_h, ld_dh, ld_dx;
    int32_t kind, dt, w_dt, reserved;
} fp8_norm_bwd_t;
FP8_API fp8_status_t fp8_norm_bwd(fp8_ctx *ctx, const fp8_norm_bwd_t *args, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FP8_NORM_H */
