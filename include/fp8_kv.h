/*
 * fp8_kv.h -- paged FP8 key/value cache and the attention that reads it, for inference with the FP8 linears of
 * fp8lin.h (the conventions stated there hold here too: status codes, device pointers, streams, no allocation, no
 * synchronisation, argument errors returned before anything is launched).
 *
 * The paper quantises the linears only (Section 3.1 for inference) and has no counterpart for the cache between the
 * QKV matmul and the output matmul.  Its scaling bias carries over directly: a ROW -- the head_dim numbers of one
 * token and one key/value head -- is the unit here, so that a row can be quantised the moment it exists (its amax is
 * in registers, there is no second pass over memory) and never again:
 *     bias  = floor(log2(max_num / amax)) as in Eq. 3, limited to -127 .. 64 (below an amax of 2^-57 a row is quantised
 *             under 64); 0 for a row of zeros
 *     byte  = RNE_E4(x * 2^(bias + delta)), saturating, exactly as fp8_cast_e4 with that bias
 *     number read back = native(byte) * 2^-(bias + delta),   delta = 1 under FP8_CONV_PAPER, else 0.
 * Under FP8_CONV_PAPER the largest byte is 448 for the paper's 480: rows whose amax lies in (232, 240] times a power of two
 * clip and raise FP8_FLAG_SATURATED, about one row in twenty of ordinary data, so the flag says little for such a cache.
 * Under FP8_CONV_NATIVE no finite row clips.
 * A row that holds an infinity or a NaN is cast under bias 0 and marked with the bias FP8_KV_BIAS_NONFINITE
 * (FP8_FLAG_NONFINITE_AMAX is raised): it reads back as cast, and the attention of every query that sees the row, and
 * of no other, gives NaN.
 */
#ifndef FP8_KV_H
#define FP8_KV_H

#include "fp8lin.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FP8_KV_BIAS_NONFINITE (-128)
#define FP8_KV_BIAS_MAX 64

/* Sticky device status bit, beside those of fp8lin.h: a page number outside the cache, or a length that contradicts
 * the bounds given on the host, was met, or a row that belongs to no sequence.  No access out of range was made: nothing is
 * written to such a page, its tokens read back as zeros, queries that see them give NaN.  Of a sequence beyond its bounds
 * the rows from max_q_len and the tokens from max_kv_len on are left out; the others keep their places.  Rows that are left
 * out, and rows of no sequence, are not cached, read back as zeros, and attend to nothing (zeros, lse -infinity). */
#define FP8_FLAG_BAD_INDEX 16u

/* The cache of one layer: `pages` pages, each holding page_size tokens of every key/value head.
 *   k8, v8   E4 bytes; a page is [kv_heads][page_size][head_dim], contiguous, pages page_stride bytes apart
 *   bk, bv   scaling biases; a page is [kv_heads][page_size], contiguous, pages bias_stride bytes apart
 * page_size 16, 32, 64 or 128; head_dim 64 or 128; all four pointers and both strides multiples of 16 (strides may be
 * larger than a page, e.g. where keys and values of a page share one buffer); pages * page_size < 2^31. */
typedef struct {
    uint8_t *k8, *v8;
    int8_t *bk, *bv;
    int64_t page_stride, bias_stride;
    int32_t pages, kv_heads, page_size, head_dim;
} fp8_kv_cache_t;

/* The sequences of one call.  Their new tokens lie one after the other in the rows of q, k, v and out:
 *   d_q_start     device int32 [seqs + 1], non-decreasing: sequence b has rows d_q_start[b] .. d_q_start[b+1] - 1
 *                 (possibly none)
 *   d_kv_len      device int32 [seqs]: tokens of the sequence in the cache, its new ones included; the new tokens are
 *                 the last of them: row d_q_start[b] + i is token d_kv_len[b] - (rows of b) + i
 *   d_page_table  device int32, rows table_stride apart: page of tokens page_size * p .. page_size * (p + 1) - 1 at index p;
 *                 every row, the last one too, has ceil(max_kv_len / page_size) entries
 *   tokens        rows of q, k, v and out, at least one
 *   max_q_len     bound of the rows of one sequence;  max_kv_len  bound of d_kv_len.  Both bound the launch, so tight
 *                 values cost least; of sequences beyond them the rest is left out (FP8_FLAG_BAD_INDEX). */
typedef struct {
    const int32_t *d_q_start, *d_kv_len, *d_page_table;
    int64_t table_stride;
    int32_t seqs, tokens, max_q_len, max_kv_len;
} fp8_seq_batch_t;

/* Quantise the new tokens' keys and values into the cache (one launch).
 *   k, v   [tokens][kv_heads][head_dim] of dtype dt (FP8_BF16, FP8_F16, FP8_F32), rows ld_k / ld_v elements apart, heads
 *          contiguous: the K and V columns of the QKV matmul's output as they lie.  16-byte aligned, strides multiples
 *          of 16 bytes.
 * Tokens whose position is negative (more rows than d_kv_len) are left out.  FP8_FLAG_NONFINITE_AMAX, FP8_FLAG_ZERO_AMAX
 * and FP8_FLAG_SATURATED are raised as fp8_cast_e4 raises them, per row. */
FP8_API fp8_status_t fp8_kv_append(fp8_ctx *ctx, const fp8_kv_cache_t *cache, const fp8_seq_batch_t *batch, const void *k,
                                   const void *v, fp8_dtype_t dt, int64_t ld_k, int64_t ld_v, fp8_conv_t conv,
                                   void *stream);

/* The inverse: the numbers that the cache holds for the last (d_q_start[b+1] - d_q_start[b]) of the first d_kv_len[b]
 * tokens of every sequence, so any range of a sequence can be asked for (all of it: d_q_start the running sum of
 * d_kv_len).  k, v: out, layout and alignment as in fp8_kv_append, each rounded once to dt; NULL for what is not wanted
 * (at least one).  Rows of tokens with a negative position are written as zeros. */
FP8_API fp8_status_t fp8_kv_read(fp8_ctx *ctx, const fp8_kv_cache_t *cache, const fp8_seq_batch_t *batch, void *k, void *v,
                                 fp8_dtype_t dt, int64_t ld_k, int64_t ld_v, fp8_conv_t conv, void *stream);

/* Attention of the new tokens over the cached ones, query head h reading key/value head h / (q_heads / kv_heads):
 *     out[r, h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale * q[r, h] . k_j),
 * j over the d_kv_len[b] cached tokens of the row's sequence, with causal != 0 only over those up to the row's own.
 * K and V are the numbers of fp8_kv_read.  Sums and softmax statistics are FP32.  What enters the products:
 *   up to 16 query rows per key/value head (max_q_len * q_heads / kv_heads): a query row as fp16 under a power of two (exact
 *     for numbers down to 2^-28 of the row's largest); a weight p_j with 16 bits
 *   more rows: a query row as two 8-bit floats under a power of two (exact down to 2^-13 of the row's largest, within 2^-21
 *     of the largest below that); a weight with 11 bits, off by 2^-10 of itself at most, by nothing on average and
 *     where its bits suffice (one token, equal scores)
 * Results are finite wherever the formula's are within bf16's range; in sequences with values of 2^49 and more, weights below
 * 2^-77 of the largest may be lost.
 *   q      [tokens][q_heads][head_dim] bf16, rows ld_q elements apart, heads contiguous
 *   out    [tokens][q_heads][head_dim] bf16, rows ld_o elements apart
 *   d_lse  NULL, or out float [tokens][q_heads]: ln sum_j p_j (what joining with attention over other keys needs)
 * A row that sees no token gives zeros and -infinity.  A query row with an infinity or a NaN gives NaN.
 * Sequences have at most 2^30 tokens, also where max_kv_len is larger.
 * q_heads a multiple of kv_heads; q and out 16-byte aligned, ld_q and ld_o multiples of 8.  Calls that share one
 * fp8_ctx must not overlap on the device, like decode-size matmuls (long contexts are split across SMs and joined in
 * the context's workspace); they follow each other on one stream like any calls. */
FP8_API fp8_status_t fp8_attn_paged(fp8_ctx *ctx, const fp8_kv_cache_t *cache, const fp8_seq_batch_t *batch, const void *q,
                                    int64_t ld_q, int32_t q_heads, void *out, int64_t ld_o, float *d_lse, float scale,
                                    int32_t causal, fp8_conv_t conv, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FP8_KV_H */
