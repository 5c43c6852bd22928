// What the attention kernels over the paged FP8 cache share.
//
// The mathematics.  With b_j, d_j the scaling biases of token j's key and value row (delta added), K8, V8 the numbers
// of their bytes and c = scale * log2(e), a row of queries q needs
//     s_j = c 2^-b_j (q . K8_j),   out = sum_j 2^s_j 2^-d_j V8_j / sum_j 2^s_j.
// The matrix instructions read K8 and V8, so the power of two of a value row is taken into the weight that multiplies
// it: with w_j = s_j - d_j and any M,
//     out = sum_j p_j V8_j / sum_j p_j 2^d_j,   p_j = 2^(w_j - M),
// exactly.  M follows the running maximum of w (not of s): p_j, which is rounded to fp16 for the product with V8 (whose
// bytes are fp16 numbers exactly), then keeps its 11 bits wherever its product matters, however different the rows'
// biases are.  M is chosen 7 below the maximum and moved only when a w exceeds M + 15, so that moving it (and rescaling
// what has been summed) is rare; p_j stays below 2^15 and is resolved down to 2^-31 of the largest weight.
// The denominator is summed in FP32 from the same p_j.  (Rows of one sequence whose biases lie more than 120 apart, that
// is values 2^120 times each other, are beyond what its range resolves.)
#pragma once

#include "kv_common.cuh"

namespace fp8lin {

struct AttnParams {
    KvParams kv;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    float *part;          // workspace of partial results (ctx->d_partial)
    unsigned *count;      // arrival counters (ctx->d_attn_count), zero between calls
    int64_t ld_q, ld_o;
    int32_t q_heads, group, causal;
    float c;              // scale * log2(e)
};

constexpr float kNoMax = -3.0e38f;    // "no token yet": finite, so that 2^(-inf - M) is 0 and not NaN
constexpr float kLift = 7.0f;         // M = maximum - kLift ...
constexpr float kSlack = 15.0f;       // ... until a weight exceeds M + kSlack
constexpr float kLn2 = 0.693147180559945309f;

#ifdef __CUDACC__

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_approx(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two E4 bytes each of the low and the high half of a word as fp16 pairs (exact).
__device__ __forceinline__ void e4_to_f16(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint4 ldg_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg_stream2(const void *p)
{
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

// 2^-(b + delta) of a key row, NaN for a row marked non-finite.
__device__ __forceinline__ float key_factor(int b, int delta)
{
    return b == FP8_KV_BIAS_NONFINITE ? __int_as_float(0x7FFFFFFF) : pow2_normal(min(126, -(b + delta)));
}

// A sequence's lengths, cut to the bounds of the launch.
struct SeqShape {
    int first, n, len;
};
__device__ __forceinline__ SeqShape seq_shape(const KvParams &kv, int b, bool &cut)
{
    SeqShape s;
    s.first = __ldg(kv.q_start + b);
    s.n = __ldg(kv.q_start + b + 1) - s.first;
    s.len = __ldg(kv.kv_len + b);
    cut = s.len < 0 || s.len > kv.max_kv_len || s.n < 0 || s.n > kv.max_q_len || s.first < 0 || s.first > kv.tokens ||
          s.n > kv.tokens - s.first;
    if (cut) {
        s.len = min(max(s.len, 0), kv.max_kv_len);
        s.n = min(max(s.n, 0), kv.max_q_len);
        if (s.first < 0 || s.first > kv.tokens) s.n = 0;
        else s.n = min(s.n, kv.tokens - s.first);
    }
    return s;
}

#endif
}  // namespace fp8lin
