// What the attention kernels over the paged FP8 cache share.
//
// The mathematics.  With b_j, d_j the scaling biases of token j's key and value row (delta added), K8, V8 the numbers
// of their bytes and c = scale * log2(e), a row of queries q needs
//     s_j = c 2^-b_j (q . K8_j),   p_j = 2^(s_j - M),   out = sum_j p_j (2^-d_j V8_j) / sum_j p_j.
// M is the row's maximum when it was last looked at: it moves only when a score lies far above it, so that rescaling what
// has been summed is rare.  FP32 has the room for weights up to 2^60 as long as values stay below 2^49.  From the first tokens
// on that hold larger ones (kLargeValue) M is kept above the maximum by so much that the weights' sum stays below 1, and sums
// of weights and values are finite wherever the result is; of such a sequence's weights those below about 2^-77 (2^30
// tokens) to 2^-100 (a few hundred) of the largest are lost.  Statistics and sums are FP32.  A value 2^-d V8 has four significant bits, so
// it is a bf16 or tf32 number exactly; how a weight p is held for the second product each kernel says.
#pragma once

#include "kv_common.cuh"

namespace fp8lin {

struct AttnParams {
    KvParams kv;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    float *part;          // workspace of partial results (ctx->d_partial)
    unsigned long long *count;   // the call's set of arrival counters (ctx->d_attn_count)
    unsigned call;               // the call's number
    int64_t ld_q, ld_o;
    int32_t q_heads, group, causal;
    int32_t row_tiles, min_share;   // chunk kernel: units of the longest sequence per head; least steps of a CTA
    float c;              // scale * log2(e)
};

// A score is (q 2^e . K8) (2^-b) (|c| 2^-e), each factor a power of two but for c.  The first product is below 2^32; a key factor is
// up to 2^126 and would take it out of FP32 where keys are large and queries small, so kKeyLift powers of two of the key
// factor (2^-65 and more) go to the query's.
constexpr int kKeyLift = 36;

constexpr int kLargeValue = -40;      // values cast under a bias (delta added) below this may reach 2^49
constexpr float kNoMax = -3.0e38f;    // M before the first token: finite, so that 2^(-inf - M) is 0 and not NaN
constexpr float kLn2 = 0.693147180559945309f;

#ifdef __CUDACC__

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^-b for the keys cast under bias b (delta added), 2^-kKeyLift of it
__device__ __forceinline__ float key_factor(int b) { return pow2_normal(min(126, -b) - kKeyLift); }
// c 2^-e with the keys' powers of two, for e from -120 to 126; finite, so that a score of 0 stays 0
__device__ __forceinline__ float query_factor(float c, int e)
{
    const int n = kKeyLift - e;
    const float x = c * pow2_normal(min(n, 100)) * pow2_normal(max(n - 100, 0));
    return fminf(fmaxf(x, -3.402823466e38f), 3.402823466e38f);
}
__device__ __forceinline__ float log2_approx(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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

// Arrivals of this call at a counter before this one.  A counter holds the number of the call that it counts for above the
// arrivals: what other calls left there (a call that gave up waiting, calls that overlapped against their contract) counts as
// nothing, so it spoils no later call.  Counters are left at 0, so the usual arrival is two atomics of which only the second
// one's result is waited for (one comparing swap that repeats until it succeeds: 16.8 instead of 10.0 us where 16 CTAs arrive
// at once, one token on 1009).
__device__ __forceinline__ unsigned arrive(unsigned long long *counter, unsigned call)
{
    const unsigned long long none = (unsigned long long)call << 32;
    atomicCAS(counter, 0ull, none);
    unsigned long long old = atomicAdd(counter, 1ull);
    while ((unsigned)(old >> 32) != call) {      // something was left here: the first to replace it is the first arrival
        const unsigned long long seen = __ldcg(counter);
        if ((unsigned)(seen >> 32) == call) old = atomicAdd(counter, 1ull);
        else if (atomicCAS(counter, seen, none + 1u) == seen) return 0u;
    }
    return (unsigned)old;
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

// A sequence's lengths, cut to the bounds of the launch, and the place of its first row: token pos of the sequence, from the
// lengths as they were, so that a row of a sequence that was cut still sees what the cache has up to the row's own token.
struct SeqShape {
    int first, n, len, pos;
};
// tokens that the sequence's row i sees
__device__ __forceinline__ int tokens_seen(const SeqShape &s, int causal, int i)
{
    return causal ? min(s.len, max(0, s.pos + i + 1)) : s.len;
}
// cut: something was cut, or rows before the first sequence or behind the last belong to none
__device__ __forceinline__ SeqShape seq_shape(const KvParams &kv, int b, bool &cut)
{
    SeqShape s;
    s.first = __ldg(kv.q_start + b);
    s.n = __ldg(kv.q_start + b + 1) - s.first;
    s.len = __ldg(kv.kv_len + b);
    s.pos = s.len - s.n;
    cut = s.len < 0 || s.len > kv.max_kv_len || s.n < 0 || s.n > kv.max_q_len || s.first < 0 || s.first > kv.tokens ||
          s.n > kv.tokens - s.first || (b == 0 && s.first != 0) || (b == kv.seqs - 1 && s.n != kv.tokens - s.first);
    if (cut) {
        // (sums of a place and a row stay within 32 bits: lengths and rows are at most 2^30)
        s.pos = (int)max(-(1ll << 30), min((long long)s.len - s.n, 1ll << 30));
        s.len = min(max(s.len, 0), kv.max_kv_len);
        s.n = min(max(s.n, 0), kv.max_q_len);
        if (s.first < 0 || s.first > kv.tokens) s.n = 0;
        else s.n = min(s.n, kv.tokens - s.first);
    }
    return s;
}

// Rows that no sequence has within its bounds: zeros, and -infinity as their lse.  By all warps of the grid; only called
// where something was cut.
static __device__ __noinline__ void write_left_out_rows(const KvParams &kv, uint16_t *out, int64_t ld_o, float *lse, int q_heads, int d)
{
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int64_t t = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5); t < kv.tokens; t += (int64_t)gridDim.x * warps) {
        const int b = find_sequence(kv.q_start, kv.seqs, (int)t, lane);
        bool cut;
        if (b >= 0) {
            const SeqShape s = seq_shape(kv, b, cut);
            if (t - s.first < s.n) continue;
        }
        for (int64_t i = lane * 8; i < (int64_t)q_heads * d; i += 32 * 8) *reinterpret_cast<uint4 *>(out + t * ld_o + i) = make_uint4(0, 0, 0, 0);
        if (lse)
            for (int h = lane; h < q_heads; h += 32) lse[t * q_heads + h] = -INFINITY;
    }
}

#endif
}  // namespace fp8lin
