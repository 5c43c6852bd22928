// Attention over the paged FP8 cache.
//
// One CTA per query row (token, head): a thread takes every 128th cached token, holds its score, and the CTA keeps the
// running maximum and sum of the softmax (statistics and sums in FP32) over blocks of 128 tokens.
#include "attn_common.cuh"

namespace fp8lin {

fp8_status_t attn_decode(const fp8_ctx *ctx, const AttnParams &p, int head_dim, int rows, cudaStream_t st);   // attn_decode.cu

__device__ __forceinline__ float e4_number(uint8_t c)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    float f;
    asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.f32.f16 %0, lo; }" : "=f"(f) : "r"(h));
    return f;
}

__device__ __forceinline__ float block_reduce(float v, bool take_max, float *s)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float w = __shfl_xor_sync(0xFFFFFFFFu, v, o);
        v = take_max ? fmaxf(v, w) : v + w;
    }
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = take_max ? fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) : (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return v;
}

template <int D>
__global__ void __launch_bounds__(128) attn_row_kernel(const AttnParams p)
{
    __shared__ float q[D], w[128], red[4];
    const KvParams &kv = p.kv;
    const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31;
    const int b = find_sequence(kv.q_start, kv.seqs, t, lane);
    if (b < 0) return;
    const int first = __ldg(kv.q_start + b), n = __ldg(kv.q_start + b + 1) - first;
    int len = __ldg(kv.kv_len + b);
    if (threadIdx.x == 0 && (len < 0 || len > kv.max_kv_len || n > kv.max_q_len)) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    if (t - first >= kv.max_q_len) return;
    const int64_t last = (int64_t)len - n + (t - first);
    len = min(max(len, 0), kv.max_kv_len);
    if (p.causal) len = (int)min((int64_t)len, max((int64_t)0, last + 1));
    const int hk = head / p.group;
    for (int i = threadIdx.x; i < D; i += 128)
        q[i] = __uint_as_float((uint32_t)p.q[t * p.ld_q + (int64_t)head * D + i] << 16) * (p.c * kLn2);
    __syncthreads();
    bool q_bad = false;
    for (int i = 0; i < D; ++i) q_bad |= !(fabsf(q[i]) < INFINITY);
    float m = -INFINITY, l = 0.0f, acc = 0.0f;
    for (int j0 = 0; j0 < len; j0 += 128) {
        const int j = j0 + threadIdx.x;
        float s = -INFINITY;
        if (j < len) {
            const int page = __ldg(kv.table + (int64_t)b * kv.table_stride + (j >> kv.page_shift));
            if ((unsigned)page >= (unsigned)kv.pages) {
                raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
                s = NAN;
            } else {
                const int64_t row = ((int64_t)hk << kv.page_shift) + (j & ((1 << kv.page_shift) - 1));
                const uint8_t *kr = kv.k8 + page * kv.page_stride + row * D;
                float dot = 0.0f;
                for (int i = 0; i < D; ++i) dot = fmaf(q[i], e4_number(kr[i]), dot);
                const int bk = kv.bk[page * kv.bias_stride + row], bv = kv.bv[page * kv.bias_stride + row];
                s = q_bad || bk == FP8_KV_BIAS_NONFINITE || bv == FP8_KV_BIAS_NONFINITE ? NAN : dot * pow2_normal(-(bk + kv.delta));
            }
        }
        const float top = fmaxf(m, block_reduce(s, true, red));
        const float base = top == -INFINITY ? 0.0f : top, shrink = __expf(m - base);
        const float pj = __expf(s - base);
        l = l * shrink + block_reduce(pj, false, red);
        w[threadIdx.x] = pj;
        __syncthreads();
        acc *= shrink;
        m = top;
        if (threadIdx.x < D) {
            for (int jj = 0; jj < min(128, len - j0); ++jj) {
                const int page = __ldg(kv.table + (int64_t)b * kv.table_stride + ((j0 + jj) >> kv.page_shift));
                if ((unsigned)page >= (unsigned)kv.pages) { acc = NAN; continue; }
                const int64_t row = ((int64_t)hk << kv.page_shift) + ((j0 + jj) & ((1 << kv.page_shift) - 1));
                const int bv = kv.bv[page * kv.bias_stride + row];
                acc = fmaf(w[jj] * pow2_normal(-(applied_bias(bv) + kv.delta)), e4_number(kv.v8[page * kv.page_stride + row * D + threadIdx.x]), acc);
            }
        }
        __syncthreads();
    }
    if (threadIdx.x < D) {
        const float o = l == 0.0f ? 0.0f : acc / l;
        uint32_t h;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(0.0f), "f"(o));
        p.out[t * p.ld_o + (int64_t)head * D + threadIdx.x] = (uint16_t)h;
    }
    if (p.lse && threadIdx.x == 0) p.lse[(int64_t)t * p.q_heads + head] = l == 0.0f ? -INFINITY : m + logf(l);
}

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
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.lse = d_lse;
    p.ld_q = ld_q;
    p.ld_o = ld_o;
    p.part = ctx->d_partial;
    p.count = ctx->d_attn_count;
    p.q_heads = q_heads;
    p.group = q_heads / c->kv_heads;
    p.causal = causal != 0;
    p.c = scale * 1.44269504088896341f;
    const int64_t rows = (int64_t)batch->max_q_len * p.group;
    if (rows <= 16) return attn_decode(ctx, p, c->head_dim, (int)rows, (cudaStream_t)stream);
    const dim3 grid((unsigned)batch->tokens, (unsigned)q_heads);
    count_launch();
    if (c->head_dim == 128) attn_row_kernel<128><<<grid, 128, 0, (cudaStream_t)stream>>>(p);
    else attn_row_kernel<64><<<grid, 128, 0, (cudaStream_t)stream>>>(p);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

}  // extern "C"
