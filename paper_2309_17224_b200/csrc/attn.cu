// Entry point of the attention over the paged FP8 cache: checks of the arguments, and which kernel takes the call.
#include "attn_common.cuh"

namespace fp8lin {

fp8_status_t attn_decode(const fp8_ctx *ctx, const AttnParams &p, int head_dim, int rows, cudaStream_t st);   // attn_decode.cu
fp8_status_t attn_chunk(const fp8_ctx *ctx, const AttnParams &p, const fp8_kv_cache_t *c, cudaStream_t st);   // attn_chunk.cu

}  // namespace fp8lin

extern "C" {

fp8_status_t fp8_attn_paged(fp8_ctx *ctx, const fp8_kv_cache_t *c, const fp8_seq_batch_t *batch, const void *q, int64_t ld_q,
                            int32_t q_heads, void *out, int64_t ld_o, float *d_lse, float scale, int32_t causal, fp8_conv_t conv,
                            void *stream)
{
    using namespace fp8lin;
    const fp8_status_t s = check_kv(ctx, c, batch, (int)conv);
    if (s != FP8_OK) return s;
    if (!q || !out) return FP8_ERR_NULL;
    if (q_heads <= 0 || q_heads % c->kv_heads != 0) return FP8_ERR_SHAPE;
    if (ld_q < (int64_t)q_heads * c->head_dim || ld_o < (int64_t)q_heads * c->head_dim) return FP8_ERR_SHAPE;
    if (!(fabsf(scale) <= 3.402823466e38f)) return FP8_ERR_SHAPE;
    if (!kv_aligned16(q) || !kv_aligned16(out) || ld_q % 8 != 0 || ld_o % 8 != 0 || (reinterpret_cast<uintptr_t>(d_lse) & 3u))
        return FP8_ERR_ALIGN;
    AttnParams p;
    p.kv = make_kv_params(ctx, c, batch, (int)conv);
    // sums of a length and a row's place then stay within 32 bits (2^30 tokens of one head are 128 GB of cache)
    if (p.kv.max_kv_len > 1 << 30) p.kv.max_kv_len = 1 << 30;
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.lse = d_lse;
    p.ld_q = ld_q;
    p.ld_o = ld_o;
    p.part = ctx->d_partial;
    p.q_heads = q_heads;
    p.group = q_heads / c->kv_heads;
    p.causal = causal != 0;
    p.c = scale * 1.44269504088896341f;
    const int64_t rows = (int64_t)batch->max_q_len * p.group;
    if (rows > (int64_t)1 << 30) return FP8_ERR_SHAPE;
    // Every call counts arrivals under a number of its own.  A captured call has the same number in every replay, so captured
    // calls have sets of counters of their own too, which no other call leaves anything in.
    cudaStreamCaptureStatus capture;
    if (cudaStreamIsCapturing((cudaStream_t)stream, &capture) != cudaSuccess) return FP8_ERR_CUDA;
    const unsigned set = capture == cudaStreamCaptureStatusNone ? 0u : 1u + ctx->attn_captured++ % (kAttnSets - 1);
    p.count = ctx->d_attn_count + (size_t)set * kAttnCounters;
    p.call = ++ctx->attn_calls;
    // At most 16 query rows per key/value head: the kernel whose instructions take 8 or 16 rows; more: tiles of 128.  Few rows
    // / chunks, us from a graph, 16 sequences on up to 4096 tokens: 1 row (8/8 heads) 35 / 73, 8 rows (64/8) 36 / 75, 16 rows
    // (64/4) 30 / 46 and (64/8, two tokens) 51 / 81; 24 rows (three tokens) 83 by chunks.
    if (rows <= 16) return attn_decode(ctx, p, c->head_dim, (int)rows, (cudaStream_t)stream);
    return attn_chunk(ctx, p, c, (cudaStream_t)stream);
}

}  // extern "C"
