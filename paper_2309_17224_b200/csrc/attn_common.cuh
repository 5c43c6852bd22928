// What the attention kernels over the paged FP8 cache share.
//
// The mathematics.  With b_j, d_j the scaling biases of token j's key and value row (delta added), K8, V8 the numbers
// of their bytes and c = scale * log2(e), a row of queries q needs
//     s_j = c 2^-b_j (q . K8_j),   p_j = 2^(s_j - M),   out = sum_j p_j (2^-d_j V8_j) / sum_j p_j.
// M is the row's maximum when it was last looked at: it moves only when a score exceeds it by more than kSlack, so that
// rescaling what has been summed is rare (p_j stays below 2^kSlack, and FP32 has room below).
// The second product runs on bf16: a value 2^-d V8 has four significant bits, so it is a bf16 number exactly, and a
// weight is the sum of two, p = p1 + p2, p1 the leading eight bits and p2 the rest rounded to eight: sixteen bits at any
// size.  One bf16 (2^-9 of every weight) would be coarser than the rounding of the output itself; fp16 would do for
// weights near the maximum but has none left below 2^-39 of it, and those count in dimensions where the tokens above
// them hold zeros.  The denominator is the FP32 sum of the unrounded p_j.
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
    int32_t row_tiles, min_share;   // chunk kernel: units of the longest sequence per head; least steps of a CTA
    float c;              // scale * log2(e)
};

constexpr float kNoMax = -3.0e38f;    // M before the first token: finite, so that 2^(-inf - M) is 0 and not NaN
constexpr float kSlack = 40.0f;       // M is moved when a score exceeds it by more
constexpr float kSumLimit = 1.152921504606847e18f;   // 2^60: the same, seen in the sum of the weights
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

// E4 bytes as bf16: the exponent and mantissa fields moved to where bf16 has them give the number times 2^-120 (also for
// the subnormals of E4), which the multiplication by 2^(120 - d) mends and scales at once, exactly.
//   spread: a word whose bytes 1 and 3 hold the two E4 bytes (bytes 0 and 2 are ignored)
__device__ __forceinline__ uint32_t e4_fields_as_bf16(uint32_t spread) { return ((spread >> 4) & 0x07F007F0u) | (spread & 0x80008000u); }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t x, uint32_t y)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// 2^(120 - d) as a bf16 number; for d < -7 that is beyond bf16 and the rest, 2^(-7 - d), is a second factor.
__device__ __forceinline__ uint32_t value_factor(int d) { return (uint32_t)(247 - max(d, -7)) << 7; }
__device__ __forceinline__ uint32_t value_factor_rest(int d) { return (uint32_t)(127 + max(-7 - d, 0)) << 7; }

// p = p1 + p2 for two weights: the upper halves as they are, the rest rounded.
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &p1, uint32_t &p2)
{
    p1 = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    p2 = pack_bf16x2(a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), b - __uint_as_float(__float_as_uint(b) & 0xFFFF0000u));
}

// Four dimensions of a row's sum under the running M of the parts joined so far.
struct JoinedRow {
    float4 v;
    float m, l;
};
__device__ __forceinline__ void join_start(JoinedRow &a)
{
    a.v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    a.m = kNoMax;
    a.l = 0.0f;
}
__device__ __forceinline__ void join_part(JoinedRow &a, float m, float l, float4 y)
{
    const float top = fmaxf(a.m, m), f = exp2_approx(a.m - top), g = exp2_approx(m - top);
    a.v.x = fmaf(y.x, g, a.v.x * f);
    a.v.y = fmaf(y.y, g, a.v.y * f);
    a.v.z = fmaf(y.z, g, a.v.z * f);
    a.v.w = fmaf(y.w, g, a.v.w * f);
    a.l = fmaf(l, g, a.l * f);
    a.m = top;
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
