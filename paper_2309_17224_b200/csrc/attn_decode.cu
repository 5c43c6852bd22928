// Attention over the paged FP8 cache for few query rows: at most 16 rows share a key/value head (one new token with up
// to 16 query heads per key/value head, or a few tokens with fewer).
//
// Bound by the cache's bytes.  Every byte goes from global memory into the registers of the lane that feeds it to the
// matrix instruction: no shared memory on the way, no barrier, no swizzle.  A warp takes blocks of 16 tokens (never
// across a page); tokens are the rows of the first product and head dimensions the rows of the second, queries are the
// columns of both (m16n8k16, 16-bit operands, FP32 sums), so eight queries cost one instruction and none is padded to 16:
//   S^T[16 tokens x 8 rows] = K[16 x D] Q^T:   lane (g = lane / 4, t = lane % 4) holds 16 contiguous bytes of tokens g and
//       g + 8 per 64 dimensions; which dimension meets which contraction index is free as long as Q agrees, so the
//       bytes are used in memory order (K as fp16, one conversion per two bytes; a query row as fp16 under a power of two)
//   O^T[D x 8 rows] += V^T P^T:   lane (g, t) holds 16 contiguous dimensions of tokens 2t, 2t+1, 2t+8, 2t+9; a byte
//       permute brings two tokens together, five instructions make a bf16 pair.  P^T, in its two terms, comes out of
//       S^T by 8x8 transposes (movmatrix).
// A warp holds one block: its keys' registers are requested again (the next block's) as soon as the first product is done,
// its values' after the second.  (Together with the join's many loads in flight this took 16 sequences on 4096 from 40.2 us,
// with two blocks per warp, to 35.8.)  CTAs per SM (decode_ctas) are as many as the registers allow without a spill: up to 8
// rows three of 168 registers for 128 dimensions (four of 128 spill 84 bytes: 16 sequences on 4096 36.9 against 35.7 us, 64 on
// 512 28.1 against 26.2) and four of 128 for 64 dimensions (three: 32/32 heads, 16 on 4096, 72 against 64 us); up to 16 rows
// two of 254 and 189.  The blocks of all (sequence,
// head) units form one list, cut evenly between the CTAs (a sequence's length changes nothing in the balance); a unit that
// lies in several CTAs leaves partial sums in the workspace, joined in order by the CTA that arrives last, so results do
// not depend on the order of arrival.
// Measured from a graph (64/8 heads of 128): 16 ragged sequences on up to 4096 tokens 35.4 us for 109 MB (17 us at the
// measured copy rate), on up to 16384 95 us for 435 MB.  Longer contexts add 5.45 TB/s; about 15 us are fixed: launch, lookup,
// first loads, changes of unit, and the join (2.6 us, taken at four CTAs per SM).
#include <type_traits>

#include "attn_common.cuh"

namespace fp8lin {

constexpr int kDecodeWarps = 4;
constexpr int kDecodeThreads = 32 * kDecodeWarps;
constexpr int kBlockTokens = 16;
constexpr int decode_ctas(int d, int nt) { return nt > 1 ? 2 : d == 128 ? 3 : 4; }

// M is moved when a score exceeds it by more than kSlack, to that score.  Once values are large no weight may be above a
// quarter divided by the number of tokens: M is moved when a score comes closer to it than that, to kLargeLift further away.
constexpr float kSlack = 40.0f, kLargeLift = 8.0f;

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint2 load_stream2(const void *p)
{
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
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

// A weight as the sum of two bf16 numbers, p = p1 + p2 (two weights at a time): p1 the leading eight bits as they are, p2 the
// rest rounded to eight, sixteen bits at any size.  One bf16 (2^-9 of every weight) would be coarser than the rounding of
// the output itself; fp16 would do for weights near the maximum but has none left below 2^-39 of it, and those count in
// dimensions where the tokens above them hold zeros.
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &p1, uint32_t &p2)
{
    p1 = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    p2 = pack_bf16x2(a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), b - __uint_as_float(__float_as_uint(b) & 0xFFFF0000u));
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// One block's bytes as a lane holds them.
template <int D>
struct KvBlock {
    static constexpr int kKChunks = D / 64;
    static constexpr int kVWords = D / 32;       // words of each of the four value rows
    uint32_t k[2][kKChunks][4];
    uint32_t v[4][kVWords];
    int bk[2], bv[2];
    int bad;                                     // the block's page number is out of range
};

template <int D>
__device__ __forceinline__ void load_k(KvBlock<D> &x, const uint8_t *k, const int8_t *bk, const int8_t *bv, int g, int t)
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int i = 0; i < KvBlock<D>::kKChunks; ++i) {
            const uint4 w = load_stream(k + (g + 8 * r) * D + (t + 4 * i) * 16);
            x.k[r][i][0] = w.x; x.k[r][i][1] = w.y; x.k[r][i][2] = w.z; x.k[r][i][3] = w.w;
        }
        x.bk[r] = bk[g + 8 * r];
        x.bv[r] = bv[g + 8 * r];
    }
}
template <int D>
__device__ __forceinline__ void load_v(KvBlock<D> &x, const uint8_t *v, int g, int t)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint8_t *src = v + (2 * t + (r & 1) + 8 * (r >> 1)) * D + g * (D / 8);
        if constexpr (D == 128) {
            const uint4 w = load_stream(src);
            x.v[r][0] = w.x; x.v[r][1] = w.y; x.v[r][2] = w.z; x.v[r][3] = w.w;
        } else {
            const uint2 w = load_stream2(src);
            x.v[r][0] = w.x; x.v[r][1] = w.y;
        }
    }
}

// Where the CTA stands in the list of blocks: a unit (sequence b, head h) and the range of its blocks.
struct Unit {
    int b, h;
    SeqShape s;
    int blocks;           // of the whole unit, at least one where the sequence has rows
    int64_t first_block;  // of the unit, in the list
};

__device__ __forceinline__ int unit_blocks(const SeqShape &s) { return s.n > 0 ? max(1, (s.len + kBlockTokens - 1) / kBlockTokens) : 0; }

template <int D, int NT>
__global__ void __launch_bounds__(kDecodeThreads, decode_ctas(D, NT)) attn_decode_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int kRows = 8 * NT;
    constexpr int kPart = kRows * (D + 2);       // floats of a partial result
    __shared__ __align__(16) float s_o[kDecodeWarps][kRows][D];
    __shared__ float s_m[kDecodeWarps][kRows], s_l[kDecodeWarps][kRows];
    __shared__ unsigned s_last;
    const KvParams &kv = p.kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;

    // ---- the CTA's share of the list (every warp computes it for itself) ----
    int64_t total = 0;
    bool any_cut = false;
    for (int b0 = 0; b0 < kv.seqs; b0 += 32) {
        int n = 0;
        if (b0 + lane < kv.seqs) {
            bool cut;
            n = unit_blocks(seq_shape(kv, b0 + lane, cut));
            any_cut |= cut;
        }
        total += __reduce_add_sync(0xFFFFFFFFu, n);
    }
    if (__builtin_expect(__any_sync(0xFFFFFFFFu, any_cut), 0)) {
        if (blockIdx.x == 0 && warp == 0 && lane == 0) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
        write_left_out_rows(kv, p.out, p.ld_o, p.lse, p.q_heads, D);
    }
    total *= kv.kv_heads;
    // at least one block per warp, so that short lists are not spread over CTAs that then wait for one another's sums
    const int64_t share = max((total + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)kDecodeWarps);
    int64_t at = blockIdx.x * share;
    const int64_t end = min(total, at + share);
    if (at >= end) return;

    Unit u;
    {
        int64_t before = 0;
        for (int b0 = 0;; b0 += 32) {
            SeqShape s = {0, 0, 0, 0};
            int n = 0;
            if (b0 + lane < kv.seqs) {
                bool cut;
                s = seq_shape(kv, b0 + lane, cut);
                n = unit_blocks(s);
            }
            int64_t upto = (int64_t)n * kv.kv_heads;   // inclusive sums
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= o) upto += x;
            }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, at < before + upto);
            if (hit) {
                const int l = __ffs(hit) - 1;
                u.b = b0 + l;
                u.s.first = __shfl_sync(0xFFFFFFFFu, s.first, l);
                u.s.n = __shfl_sync(0xFFFFFFFFu, s.n, l);
                u.s.len = __shfl_sync(0xFFFFFFFFu, s.len, l);
                u.s.pos = __shfl_sync(0xFFFFFFFFu, s.pos, l);
                u.blocks = __shfl_sync(0xFFFFFFFFu, n, l);
                const int64_t start = before + __shfl_sync(0xFFFFFFFFu, upto, l) - (int64_t)u.blocks * kv.kv_heads;
                u.h = (int)((at - start) / u.blocks);
                u.first_block = start + (int64_t)u.h * u.blocks;
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }

    const int size = 1 << kv.page_shift, blocks_per_page_shift = kv.page_shift - 4;
    while (true) {
        const int lo = (int)(at - u.first_block), hi = (int)min((int64_t)u.blocks, end - u.first_block);
        const int rows = u.s.n * p.group;

        // ---- this warp's blocks: lo + warp, every fourth; the first is requested before the queries are looked at ----
        const int32_t *table = kv.table + (int64_t)u.b * kv.table_stride;
        const int mine = max(0, (hi - lo - warp + kDecodeWarps - 1) / kDecodeWarps);
        const int count = u.s.len > 0 ? mine : 0;
        int pages = 0;            // lane i: page of the warp's block (32 * round + i)
        auto fetch_pages = [&](int i0) {
            const int blk = lo + warp + (i0 + lane) * kDecodeWarps;
            pages = i0 + lane < count ? __ldg(table + (blk >> blocks_per_page_shift)) : 0;
        };
        int64_t v_at;
        auto request_k = [&](KvBlock<D> &x, int i, int64_t &v_off) {
            if ((i & 31) == 0) fetch_pages(i);
            const int page = __shfl_sync(0xFFFFFFFFu, pages, i & 31);
            const int blk = lo + warp + i * kDecodeWarps;
            x.bad = (unsigned)page >= (unsigned)kv.pages;
            const int64_t row = ((int64_t)u.h << kv.page_shift) + ((blk * kBlockTokens) & (size - 1));
            const int64_t pg = x.bad ? 0 : page;
            v_off = pg * kv.page_stride + row * D;
            const int64_t b_off = pg * kv.bias_stride + row;
            load_k<D>(x, kv.k8 + v_off, kv.bk + b_off, kv.bv + b_off, g, t);
        };
        KvBlock<D> cur;
        if (count > 0) { request_k(cur, 0, v_at); load_v<D>(cur, kv.v8 + v_at, g, t); }

        // ---- queries: fp16 under a power of two per row (exact for bf16 unless 2^28 below the row's largest) ----
        uint32_t q[NT][D / 16][2];
        float rc[NT][2];          // c / that power and the keys' share, for the rows of S^T's columns
        int limit[NT][2];         // tokens those rows see
        const int all_see = tokens_seen(u.s, p.causal, 0);    // tokens that every row sees
        {
            float mine[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int r = 8 * j + g;
                uint32_t w[D / 64][8];
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    uint4 x = make_uint4(0, 0, 0, 0), y = x;
                    if (r < rows) {
                        const uint16_t *src = p.q + (int64_t)(u.s.first + r / p.group) * p.ld_q +
                                              (int64_t)(u.h * p.group + r % p.group) * D + (t + 4 * i) * 16;
                        x = *reinterpret_cast<const uint4 *>(src);
                        y = *reinterpret_cast<const uint4 *>(src + 8);
                    }
                    w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
                    w[i][4] = y.x; w[i][5] = y.y; w[i][6] = y.z; w[i][7] = y.w;
#pragma unroll
                    for (int k = 0; k < 8; ++k) m = max(m, max((w[i][k] << 16) & 0x7FFF0000u, w[i][k] & 0x7FFF0000u));
                }
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
                // the row's largest lands in [2^14, 2^15)
                const int e = m == 0 ? 0 : max(-113, min(126, 14 + 127 - (int)(m >> 23)));
                const float f = pow2_normal(e);
                mine[j] = m >= 0x7F800000u ? __int_as_float(0x7FFFFFFF) : query_factor(p.c, e);
#pragma unroll
                for (int i = 0; i < D / 64; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        q[j][4 * i + k / 2][k & 1] = pack_f16(__uint_as_float(w[i][k] << 16) * f, __uint_as_float(w[i][k] & 0xFFFF0000u) * f);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    rc[j][k] = __shfl_sync(0xFFFFFFFFu, mine[j], (2 * t + k) * 4);
                    limit[j][k] = tokens_seen(u.s, p.causal, (8 * j + 2 * t + k) / p.group);
                }
            }
        }

        float o[NT][D / 16][4], top[NT][2], l[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int m = 0; m < D / 16; ++m) o[j][m][0] = o[j][m][1] = o[j][m][2] = o[j][m][3] = 0.0f;
            top[j][0] = top[j][1] = kNoMax;
            l[j][0] = l[j][1] = 0.0f;
        }

        // The blocks from i on; without LARGE up to the first that holds large values, whose index is returned.  (One loop
        // for both, with the margin in a register: 16 sequences on 4096 tokens 37.4 against 36.5 us at four CTAs per SM.)
        auto walk = [&](auto large_mode, int i) {
            constexpr bool kLarge = decltype(large_mode)::value;
            const float margin = (float)(34 - __clz(u.s.len));        // log2 of four times the tokens, and up to one more
            for (; i < count; ++i) {
                const int j0 = (lo + warp + i * kDecodeWarps) * kBlockTokens;
                if constexpr (!kLarge) {
                    // (marked rows and what lies behind the end are no values)
                    auto large = [&](int r) {
                        return cur.bv[r] != FP8_KV_BIAS_NONFINITE && cur.bv[r] + kv.delta < kLargeValue && j0 + g + 8 * r < u.s.len;
                    };
                    if (__builtin_expect(__any_sync(0xFFFFFFFFu, min(cur.bv[0], cur.bv[1]) < kLargeValue), 0) &&
                        __any_sync(0xFFFFFFFFu, !cur.bad && (large(0) || large(1))))
                        break;
                }
                // S^T
                float s[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.0f;
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t a0, a1, a2, a3;
                        e4_to_f16(cur.k[0][c][k], a0, a2);
                        e4_to_f16(cur.k[1][c][k], a1, a3);
#pragma unroll
                        for (int j = 0; j < NT; ++j) mma_f16(s[j], a0, a1, a2, a3, q[j][4 * c + k][0], q[j][4 * c + k][1]);
                    }
                // a page out of range is read as page 0 and then taken as non-finite
                int bk[2] = {cur.bk[0], cur.bk[1]}, bv[2] = {cur.bv[0], cur.bv[1]};
                if (cur.bad) bk[0] = bk[1] = bv[0] = bv[1] = FP8_KV_BIAS_NONFINITE;
                const int bad = cur.bad;
                // the registers of K are free: the next block's
                if (i + 1 < count) request_k(cur, i + 1, v_at);
                if (bad && lane == 0) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
                const bool marked0 = bk[0] == FP8_KV_BIAS_NONFINITE || bv[0] == FP8_KV_BIAS_NONFINITE;
                const bool marked1 = bk[1] == FP8_KV_BIAS_NONFINITE || bv[1] == FP8_KV_BIAS_NONFINITE;
                const float f0 = marked0 ? __int_as_float(0x7FFFFFFF) : key_factor(bk[0] + kv.delta);
                const float f1 = marked1 ? __int_as_float(0x7FFFFFFF) : key_factor(bk[1] + kv.delta);
                // scores; beyond what a row sees -infinity
                bool above = false;
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        s[j][k] = s[j][k] * f0 * rc[j][k];
                        s[j][2 + k] = s[j][2 + k] * f1 * rc[j][k];
                        if (j0 + kBlockTokens > all_see) {
                            if (j0 + g >= limit[j][k]) s[j][k] = -INFINITY;
                            if (j0 + g + 8 >= limit[j][k]) s[j][2 + k] = -INFINITY;
                        }
                        above |= fmaxf(s[j][k], s[j][2 + k]) > (kLarge ? top[j][k] - margin : top[j][k] + kSlack);
                    }
                if (__any_sync(0xFFFFFFFFu, above)) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float m = fmaxf(s[j][k], s[j][2 + k]);
                            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                            const float next = fmaxf(top[j][k], kLarge ? m + margin + kLargeLift : m);
                            const float shrink = exp2_approx(top[j][k] - next);
                            top[j][k] = next;
                            l[j][k] *= shrink;
#pragma unroll
                            for (int m2 = 0; m2 < D / 16; ++m2) {
                                o[j][m2][k] *= shrink;
                                o[j][m2][2 + k] *= shrink;
                            }
                        }
                }
                // p, the denominator, and P^T's two terms as the second product's operands
                uint32_t pt[NT][2][2];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        s[j][k] = exp2_approx(s[j][k] - top[j][k]);
                        s[j][2 + k] = exp2_approx(s[j][2 + k] - top[j][k]);
                        l[j][k] += s[j][k] + s[j][2 + k];
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        uint32_t p1, p2;
                        split_bf16(s[j][2 * r], s[j][2 * r + 1], p1, p2);
                        pt[j][0][r] = transpose8x8(p1);
                        pt[j][1][r] = transpose8x8(p2);
                    }
                }
                // values that no weight may meet, because 0 times a NaN is one: tokens behind the end, marked rows
                const unsigned marks = __ballot_sync(0xFFFFFFFFu, marked0), marks8 = __ballot_sync(0xFFFFFFFFu, marked1);
                if ((marks | marks8) != 0u || j0 + kBlockTokens > u.s.len) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = 2 * t + (r & 1);
                        const bool drop = ((((r >> 1) ? marks8 : marks) >> (4 * row)) & 1u) || j0 + row + 8 * (r >> 1) >= u.s.len;
                        if (drop) {
#pragma unroll
                            for (int k = 0; k < KvBlock<D>::kVWords; ++k) cur.v[r][k] = 0u;
                        }
                    }
                }
                // 2^(120 - d) of tokens 2t, 2t + 1, and of 2t + 8, 2t + 9
                const int dv0 = bv[0] + kv.delta, dv1 = bv[1] + kv.delta;
                uint32_t f_lo, f_hi, rest_lo = 0, rest_hi = 0;
                {
                    const uint32_t both = value_factor(dv0) | value_factor(dv1) << 16;
                    const uint32_t even = __shfl_sync(0xFFFFFFFFu, both, 8 * t), odd = __shfl_sync(0xFFFFFFFFu, both, 8 * t + 4);
                    f_lo = __byte_perm(even, odd, 0x5410);
                    f_hi = __byte_perm(even, odd, 0x7632);
                }
                const bool two_steps = __any_sync(0xFFFFFFFFu, min(dv0, dv1) < -7);   // values beyond 2^15
                if (two_steps) {
                    const uint32_t both = value_factor_rest(dv0) | value_factor_rest(dv1) << 16;
                    const uint32_t even = __shfl_sync(0xFFFFFFFFu, both, 8 * t), odd = __shfl_sync(0xFFFFFFFFu, both, 8 * t + 4);
                    rest_lo = __byte_perm(even, odd, 0x5410);
                    rest_hi = __byte_perm(even, odd, 0x7632);
                }
#pragma unroll
                for (int m = 0; m < D / 16; ++m) {
                    // dimensions 2m and 2m + 1 of the lane's sixteen (or eight): byte 2 (m & 1) and the next of word m / 2
                    uint32_t a[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t from = 2u * (m & 1) + (k & 1);      // byte of both tokens' words, to bytes 1 and 3
                        const uint32_t x = __byte_perm(cur.v[k & 2][m >> 1], cur.v[(k & 2) + 1][m >> 1], ((4u + from) << 12) | (from << 4));
                        a[k] = mul_bf16x2(e4_fields_as_bf16(x), k < 2 ? f_lo : f_hi);
                        if (two_steps) a[k] = mul_bf16x2(a[k], k < 2 ? rest_lo : rest_hi);
                    }
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        mma_bf16(o[j][m], a[0], a[1], a[2], a[3], pt[j][0][0], pt[j][0][1]);
                        mma_bf16(o[j][m], a[0], a[1], a[2], a[3], pt[j][1][0], pt[j][1][1]);
                    }
                }
                if (i + 1 < count) load_v<D>(cur, kv.v8 + v_at, g, t);
            }
            return i;
        };
        int done = walk(std::false_type(), 0);
        if (done < count) {
            // what was summed so far goes under an M that is as far above it
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float v = l[j][k];
                    v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
                    v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
                    v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
                    const float next = fmaxf(top[j][k], top[j][k] + log2_approx(v) + (34 - __clz(u.s.len)) + kLargeLift);
                    const float shrink = exp2_approx(top[j][k] - next);
                    top[j][k] = next;
                    l[j][k] *= shrink;
#pragma unroll
                    for (int m = 0; m < D / 16; ++m) {
                        o[j][m][k] *= shrink;
                        o[j][m][2 + k] *= shrink;
                    }
                }
            walk(std::true_type(), done);
        }
        // ---- join the warps ----
        __syncthreads();   // the previous unit's sums have been read
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v = l[j][k];
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
                const int r = 8 * j + 2 * t + k;
                if (g == 0) { s_l[warp][r] = v; s_m[warp][r] = top[j][k]; }
                float *dst = &s_o[warp][r][g * (D / 8)];
#pragma unroll
                for (int m = 0; m < D / 16; m += 2)
                    *reinterpret_cast<float4 *>(dst + 2 * m) = make_float4(o[j][m][k], o[j][m][2 + k], o[j][m + 1][k], o[j][m + 1][2 + k]);
            }
        __syncthreads();
        const bool whole = lo == 0 && hi == u.blocks;
        const int64_t first_cta = u.first_block / share, last_cta = (u.first_block + u.blocks - 1) / share;
        float *slot = p.part + ((int64_t)blockIdx.x * 2 + (lo == 0 ? 1 : 0)) * kPart;
        auto store_row = [&](int r, int d, float4 v, float m, float sum) {
            const int64_t row = u.s.first + r / p.group;
            const int head = u.h * p.group + r % p.group;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<uint2 *>(p.out + row * p.ld_o + (int64_t)head * D + d) =
                make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
            if (p.lse && d == 0)
                p.lse[row * p.q_heads + head] = sum == 0.0f ? -INFINITY : (m + log2_approx(sum)) * kLn2;
        };
        for (int idx = threadIdx.x; idx < kRows * (D / 4); idx += kDecodeThreads) {
            const int r = idx / (D / 4), d = idx % (D / 4) * 4;
            if (r >= rows) break;
            float m = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kDecodeWarps; ++w) m = fmaxf(m, s_m[w][r]);
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kDecodeWarps; ++w) {
                const float f = exp2_approx(s_m[w][r] - m);
                const float4 y = *reinterpret_cast<const float4 *>(&s_o[w][r][d]);
                v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
                sum = fmaf(s_l[w][r], f, sum);
            }
            if (whole) {
                store_row(r, d, v, m, sum);
            } else {
                *reinterpret_cast<float4 *>(slot + r * D + d) = v;
                if (d == 0) { slot[kRows * D + r] = m; slot[kRows * D + kRows + r] = sum; }
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) s_last = arrive(p.count + first_cta, p.call) == (unsigned)(last_cta - first_cta);
            __syncthreads();
            if (s_last) {
                __threadfence();
                if (threadIdx.x == 0) p.count[first_cta] = 0ull;   // a captured call comes again under its number
                // the first part lies in its CTA's slot 1 (it starts at the unit's beginning), the others in slot 0
                auto part_of = [&](int64_t c) { return p.part + (c * 2 + (c == first_cta ? 1 : 0)) * kPart; };
                // all of a thread's rows at once and four parts' loads at a time: the loads' latency is what this costs
                constexpr int kItems = kRows * (D / 4) / kDecodeThreads;
                const int d = threadIdx.x % (D / 4) * 4, r0 = threadIdx.x / (D / 4);
                constexpr int kStep = kDecodeThreads / (D / 4);
                JoinedRow sum[kItems];
#pragma unroll
                for (int k = 0; k < kItems; ++k) join_start(sum[k]);
                for (int64_t c0 = first_cta; c0 <= last_cta; c0 += 4) {
                    float m[4][kItems], l_part[4][kItems];
                    float4 y[4][kItems];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float *src = part_of(min(c0 + c, last_cta));
#pragma unroll
                        for (int k = 0; k < kItems; ++k) {
                            const int r = min(r0 + k * kStep, rows - 1);
                            m[c][k] = __ldcg(src + kRows * D + r);
                            l_part[c][k] = __ldcg(src + kRows * D + kRows + r);
                            y[c][k] = __ldcg(reinterpret_cast<const float4 *>(src + r * D + d));
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c0 + c <= last_cta) {
#pragma unroll
                            for (int k = 0; k < kItems; ++k) join_part(sum[k], m[c][k], l_part[c][k], y[c][k]);
                        }
                }
#pragma unroll
                for (int k = 0; k < kItems; ++k)
                    if (r0 + k * kStep < rows) store_row(r0 + k * kStep, d, sum[k].v, sum[k].m, sum[k].l);
            }
        }

        // ---- next unit ----
        at = u.first_block + hi;
        if (at >= end) break;
        u.first_block += u.blocks;
        if (++u.h == kv.kv_heads) {
            u.h = 0;
            do {
                ++u.b;
                bool cut;
                u.s = seq_shape(kv, u.b, cut);
                u.blocks = unit_blocks(u.s);
            } while (u.blocks == 0);
        }
    }
}

template <int D, int NT>
static fp8_status_t launch_decode(const fp8_ctx *ctx, const AttnParams &p, cudaStream_t st)
{
    const KvParams &kv = p.kv;
    // an upper bound of the list's length; CTAs beyond the blocks that there are leave at once
    const int64_t blocks = (int64_t)kv.seqs * kv.kv_heads * ((kv.max_kv_len + kBlockTokens - 1) / kBlockTokens);
    int64_t grid = (int64_t)ctx->sm_count * decode_ctas(D, NT);
    if ((blocks + kDecodeWarps - 1) / kDecodeWarps < grid) grid = (blocks + kDecodeWarps - 1) / kDecodeWarps;
    if (grid > kAttnCounters) return FP8_ERR_UNSUPPORTED;
    count_launch();
    attn_decode_kernel<D, NT><<<(unsigned)grid, kDecodeThreads, 0, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

fp8_status_t attn_decode(const fp8_ctx *ctx, const AttnParams &p, int head_dim, int rows, cudaStream_t st)
{
    if (head_dim == 128) return rows <= 8 ? launch_decode<128, 1>(ctx, p, st) : launch_decode<128, 2>(ctx, p, st);
    return rows <= 8 ? launch_decode<64, 1>(ctx, p, st) : launch_decode<64, 2>(ctx, p, st);
}

}  // namespace fp8lin
