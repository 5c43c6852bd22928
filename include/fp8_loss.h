/*
 * fp8_loss.h -- what a language model's head computes from its logits: log probabilities of given tokens with entropy and
 * the most probable tokens, and the divergence from a teacher's listed tokens, each with the gradient of the logits (the
 * conventions stated in fp8lin.h hold here too).
 *
 * The paper scores its quantised models by the log probabilities of given tokens and recovers accuracy by fine-tuning;
 * both start from the logits that the last FP8 linear leaves, and the gradient is what its E5 cast reads.
 *
 * logits: [rows][vocab] of type dt (FP8_BF16, FP8_F16, FP8_F32), rows ld elements apart, any alignment of an element.
 * With z = scale * logits (scale = 1 / temperature, positive and finite), lse = ln sum_j exp z_j, lp_j = z_j - lse,
 * p_j = exp lp_j.  Arithmetic and sums are FP32, relative to the row's largest logit.
 * A logit of -infinity is a token that cannot come: p = 0.  A row of nothing else gives lse = -infinity, entropy 0, log
 * probabilities of -infinity and a gradient of zeros.  A row with a NaN or +infinity gives NaN (and top indices of -1).
 */
#ifndef FP8_LOSS_H
#define FP8_LOSS_H

#include "fp8lin.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of the token numbers of a call. */
typedef enum { FP8_I32 = 0, FP8_I64 = 1 } fp8_itype_t;

/* What the forward calls leave for the backward ones, four floats a row:
 *   [0] the largest logit m (not scaled)   [1] ln sum_j exp(scale (x_j - m))
 *   [2] the entropy (token log probabilities only)   [3] [1] with the listed tokens left out (distillation only)
 * lse is scale * [0] + [1].  A row of nothing but -infinity has 0 and +infinity there. */
#define FP8_LOSS_SAVED 4
#define FP8_LOSS_TOP_MAX 128     /* top tokens of fp8_token_logprobs */
#define FP8_LOSS_LISTED_MAX 256  /* listed tokens a row of the distillation calls */
#define FP8_LOSS_VOCAB_MAX (1 << 20) /* vocab of the distillation calls */

/*   targets     NULL, or in, [rows] of it: the given tokens.  A negative number: none is given, logprob is 0.  A number of
 *               vocab or more raises FP8_FLAG_BAD_INDEX, logprob is NaN.
 *   logprob     NULL, or out float [rows]: lp of the given token (needs targets)
 *   entropy     NULL, or out float [rows]: -sum_j p_j lp_j
 *   lse         NULL, or out float [rows]
 *   saved       NULL, or out float [rows][4] for fp8_token_logprobs_bwd, 16-byte aligned
 *   top_k       0, or how many of the most probable tokens are wanted (at most FP8_LOSS_TOP_MAX and vocab)
 *   top_logprob, top_index    out float / it [rows][top_k], contiguous: by falling logit, equal logits by rising index.
 *               NULL together with top_k = 0.
 * At least one output. */
FP8_API fp8_status_t fp8_token_logprobs(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows,
                                        int64_t vocab, float scale, const void *targets, fp8_itype_t it, float *logprob,
                                        float *entropy, float *lse, float *saved, int32_t top_k, float *top_logprob,
                                        void *top_index, void *stream);

/* The gradient of the logits: for a row with given token t
 *     dlogits_j = scale * (g_logprob (1[j = t] - p_j) - g_entropy p_j (lp_j + entropy))
 *   g_logprob, g_entropy   in float, elements g_logprob_stride / g_entropy_stride apart (0: one number for all rows);
 *               NULL counts as zero, not both.  A row without a valid given token has no part of g_logprob.
 *   dlogits     out, of dt, rows ld_d apart; may be logits itself (ld_d = ld then).  Where its rows do not lie like those of
 *               logits relative to 16 bytes, they are written element by element.
 *   d_amax      NULL, or out: amax of dlogits (for the E5 cast of the linear below)
 * Rows whose gradients are zero are written as zeros and their logits are not read. */
FP8_API fp8_status_t fp8_token_logprobs_bwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows,
                                            int64_t vocab, float scale, const void *targets, fp8_itype_t it,
                                            const float *saved, const float *g_logprob, int64_t g_logprob_stride,
                                            const float *g_entropy, int64_t g_entropy_stride, void *dlogits, int64_t ld_d,
                                            float *d_amax, void *stream);

/* How a teacher's list stands for its distribution. */
typedef enum {
    FP8_DISTILL_TOP = 0, /* q = softmax of the listed values: the listed tokens share everything */
    FP8_DISTILL_REST = 1 /* q = exp(value), values are log probabilities; all tokens that are not listed are one more
                          * outcome with what is left, max(0, 1 - sum q) */
} fp8_distill_mode_t;

/* Divergence of the student from the teacher, per row:
 *     loss = sum_k q_k (ln q_k - lp_k)  [+ q_r (ln q_r - ln p_r) with FP8_DISTILL_REST, r: the tokens not listed]
 *   index       in, [rows][listed] of it, rows ld_index apart;  value   in float, [rows][listed], rows ld_value apart:
 *               what fp8_token_logprobs writes as top_index and top_logprob, at the same scale.  An entry with a negative
 *               index, or whose index an earlier entry of its row has, is left out; so is one with an index of vocab or
 *               more, which raises FP8_FLAG_BAD_INDEX.  Value -infinity: q = 0.
 *   loss        out float [rows].  A row without a listed token that counts has none (0).  +infinity where the student rules
 *               out a listed token with q > 0.  Where it rules out all tokens that are not listed, q_r counts as 0 (what FP32
 *               log probabilities of a complete list leave is their rounding).
 *   saved       NULL, or out float [rows][4], 16-byte aligned, for fp8_distill_bwd
 * listed 1 .. FP8_LOSS_LISTED_MAX, vocab up to FP8_LOSS_VOCAB_MAX. */
FP8_API fp8_status_t fp8_distill_fwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows,
                                     int64_t vocab, float scale, const void *index, fp8_itype_t it, int64_t ld_index,
                                     const float *value, int64_t ld_value, int32_t listed, fp8_distill_mode_t mode,
                                     float *loss, float *saved, void *stream);

/* Its gradient, g the gradient of the row's loss and Q the sum of the row's q:
 *     dlogits_j = g * scale * (Q p_j - q_j)   for listed tokens,   g * scale * p_j (Q - q_r / p_r)   for the others
 * (q_r = 0 with FP8_DISTILL_TOP); zeros where no entry counts.  p_j / p_r keeps its digits however small p_r is: where all of
 * the others carry a finite mask, too (which does not rule them out: the loss is q_r times its depth then).  g_loss, dlogits,
 * d_amax as in fp8_token_logprobs_bwd. */
FP8_API fp8_status_t fp8_distill_bwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows,
                                     int64_t vocab, float scale, const void *index, fp8_itype_t it, int64_t ld_index,
                                     const float *value, int64_t ld_value, int32_t listed, fp8_distill_mode_t mode,
                                     const float *saved, const float *g_loss, int64_t g_loss_stride, void *dlogits,
                                     int64_t ld_d, float *d_amax, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FP8_LOSS_H */
