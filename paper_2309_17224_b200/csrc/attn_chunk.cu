// Attention over the paged FP8 cache for many query rows: chunks of a prompt, drafted tokens.
//
// The query rows of one key/value head (token by token, the head's query heads side by side) are taken in tiles of 128,
// two tiles to a unit, and the cached tokens in tiles of 128, a step each; two products per pair of tiles on the
// 5th-generation tensor cores:
//   S = Q K^T   8-bit floats: the cache's key bytes are the operand as they lie (TMA, no conversion).  A query row is the sum
//               of two such numbers under one power of two, q 2^e = hi + lo: hi is e4m3, rounded to nearest, with the row's
//               largest in (224, 448]; lo is the rest.  What hi leaves of a bf16 number is at most eight units of its last
//               bit, and those have three significant bits: lo is e5m2 (an e4m3 lo ends 2^7 higher).  Together they are exact
//               down to 2^-6, 2^13 below the row's largest, and within 2^-14 below that, 2^-21 of the largest.  Two such
//               products cost what one bf16 product costs.
//   O += P V    tf32: P is left in tensor memory as the FP32 numbers that the softmax computes, in place of the scores, and
//               read from there; a value 2^-d V8 is a tf32 number exactly, four warps make them on their way into shared
//               memory (token index innermost; once for both query tiles).  The tensor cores drop P's lower thirteen
//               bits, up to 2^-10 of a weight and 2^-11.5 on average.  All weights are 1 + 2^-11.5 too large when they are
//               cut: nothing is lost on average, and a weight that has eleven bits (1, in the first place) is itself again.
//               (Half of the last kept bit added to every weight instead: 2048 tokens on 16384 1494 against 1440 us.)
//               A tf32 product costs two bf16 products; one bf16 product would be coarser than the output's rounding, two
//               (P in two bf16 terms) cost the same as tf32 and five more instructions per pair of weights (measured:
//               2048 tokens on 16384, 64/8 heads, 1675 us), and fp16 has no weights below 2^-39 of the largest.
//
// One CTA per SM holds all 512 tensor-memory columns as two slots of S / P and O.  While one slot's softmax runs, the
// other's products do.  With more than 128 rows the slots are the unit's two query tiles, with up to 128 they are the even
// and the odd steps of the one tile, added up at its end.  Within a slot the order is strict: S, softmax, O, next S; that
// also makes the rescaling of O safe without a barrier of its own, as S of a step is complete only after O of the one
// before.  The first product of the next step overwrites the weights that the second product of this one reads.  Products of
// different kinds and accumulators are not ordered by being issued one after the other, so the second product is committed
// to a barrier of the slot, and the next scores of the slot are issued only behind it.  (Halves of 64 tokens in turn within a
// slot were slower, 1736 against 1517 us in separate runs: scores of 64 columns cost the tensor cores 1.5 times their share.)
// Measured from a graph: 2048 tokens on 16384, 64/8 heads of 128, 1453 us, 709 TFLOP/s.  A step takes about 6800 cycles, its
// products 3072 of them; the softmax's chain of latencies and the waits for products and scores take the rest (before
// the wait between the second product and the next scores, and the care for large values: 1391 us).
//
// The steps of all units (query tiles of a key/value head) form one list that is cut evenly between the CTAs, whatever the
// sequences' lengths and the mask; a unit that lies in several CTAs leaves partial sums in the workspace, joined in order
// by the CTA that arrives last.
//
// Warps: 0-3 and 4-7 softmax of the two slots (one query row per thread) and output, 8-11 values, key loads and scaling
// biases, 12 the products.
#include "attn_common.cuh"
#include "ptx.cuh"

namespace fp8lin {

constexpr int kTile = 128;                 // query rows of a tile, and tokens of a step
constexpr int kKStages = 2;

constexpr int kVStages = 2;
constexpr int kChunkThreads = 32 * 13;
constexpr int kUnitRows = 2 * kTile;

template <int D>
struct ChunkShape {
    static constexpr int kQBytes = kTile * 2 * D;            // of one query tile
    static constexpr int kKBytes = kTile * D;
    static constexpr int kVBytes = kTile * D * 4;            // four blocks of [D][32 tokens]
    static constexpr int kQ = 0;                             // (the second tile's place holds the odd slot's statistics
    static constexpr int kK = kQ + 2 * kQBytes;              // where the slots share one query tile)
    static constexpr int kV = kK + kKStages * kKBytes;
    static constexpr int kScale = kV + kVStages * kVBytes;   // [3][128] floats: 2^-b of a tile's keys
    static constexpr int kLarge = kScale + 3 * kTile * 4;    // [3][4] words: whether a step's values are large, a word per warp
    static constexpr int kBar = kLarge + 3 * 16;
    static constexpr int kNumBars = 2 * kKStages + 2 * kVStages + 8 + 5 * 2 + 3;
    static constexpr int kTotal = kBar + kNumBars * 8 + 16;
    static constexpr int kDynamic = kTotal + 1024;           // slack to align the base to 1024 bytes
    static constexpr int kPart = kTile * (D + 2);            // floats of a tile's partial result: sums, M, denominators
};
constexpr uint32_t kTmemCols = 512, kTmemSlot = 256;         // per slot 128 columns of S, then P; 128 of O
// What the tensor cores cut off a weight, on average: 2^-11 E[1/m], m a mantissa in [1, 2) with its logarithm evenly spread.
// M lies log2 of 1 + this below the maximum, which makes the weights that much larger; their sum is scaled back.
constexpr float kTf32Cut = 0.7213f / 2048.0f, kTf32Kept = 1.0f / (1.0f + kTf32Cut), kTf32Lift = kTf32Cut * 1.442695f;
constexpr uint32_t kTmemO = 128;
// M is moved when the weights' sum exceeds a limit: 2^60, and once values are large 2^-10 (a unit has up to 148 parts), where M
// is put kLargeLift above the maximum and above the sum's logarithm.
constexpr float kSumLimit = 1.152921504606847e18f, kLargeSumLimit = 1.0f / 1024.0f, kLargeLift = 18.0f;

// The tensor cores' instructions take their operands from uniform registers.  So the whole warp walks the steps with
// values that the compiler can see to be uniform, and one elected lane issues: with a single lane in the loop every operand
// of every instruction was first moved over (2048 tokens on 16384: 1474 us, and the more the longer the code per
// instruction).
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r != 0;
}
// d, the descriptors' low words (HI their high ones), a's tensor-memory address, instruction descriptor
template <uint32_t A_HI, uint32_t B_HI>
__device__ __forceinline__ void chunk_mma_f8(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\n.reg .b64 da, db;\nsetp.ne.b32 p, %4, 0;\nmov.b64 da, {%1, %5};\nmov.b64 db, {%2, %6};\n"
                 "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n}\n" ::"r"(d),
                 "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(A_HI), "n"(B_HI)
                 : "memory");
}
template <uint32_t B_HI>
__device__ __forceinline__ void chunk_mma_tf32_tmem(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\n.reg .b64 db;\nsetp.ne.b32 p, %4, 0;\nmov.b64 db, {%2, %5};\n"
                 "tcgen05.mma.cta_group::1.kind::tf32 [%0], [%1], db, %3, p;\n}\n" ::"r"(d),
                 "r"(a_tmem), "r"(b), "r"(idesc), "r"(accumulate), "n"(B_HI)
                 : "memory");
}
__device__ __forceinline__ void chunk_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void chunk_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void chunk_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_load32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// Two FP32 numbers side by side: one instruction for both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void sts4(uint32_t addr, float v)
{
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(__float_as_uint(v)) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Shared-memory matrix descriptors (start address, leading and stride offsets in 16-byte units, version 1, swizzle);
// all operands here have the contraction index innermost.
//   128-byte swizzle, operand rows of 128 contiguous bytes along the contraction, groups of eight rows 1024 bytes apart
//   64-byte swizzle, rows of 64 bytes, groups of eight rows 512 bytes apart
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr >> 4) & 0x3FFFu) | 1u << 16; }
constexpr uint32_t kSw128 = (1024 >> 4) | 1u << 14 | 2u << 29, kSw64 = (512 >> 4) | 1u << 14 | 4u << 29;

__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap *map, uint32_t bar, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(y), "r"(z)
                 : "memory");
}

// A unit of the list: up to two query tiles of one key/value head.
struct ChunkUnit {
    int e;            // entry: sequence * row_tiles + place of the tiles in the sequence
    int h;
    SeqShape s;
    int row0, rows;   // first row, rows from there on
    int steps;        // tiles of tokens that any of the unit's rows sees (at least one)
    int64_t first;    // place of the unit's first step in the list
};

__device__ __forceinline__ int entry_of(const AttnParams &p, int e, SeqShape &s, int &row0, int &rows, bool &cut)
{
    const int b = e / p.row_tiles;
    s = seq_shape(p.kv, b, cut);
    row0 = (e - b * p.row_tiles) * kUnitRows;
    rows = (int)min((int64_t)s.n * p.group - row0, (int64_t)kUnitRows);
    if (rows <= 0) return 0;
    const int see = tokens_seen(s, p.causal, (row0 + rows - 1) / p.group);
    return max(1, (see + kTile - 1) / kTile);
}

// Length of the list, by a whole warp.
__device__ __forceinline__ int64_t list_length(const AttnParams &p, int lane, bool &cut)
{
    const int entries = p.kv.seqs * p.row_tiles;
    int64_t mine = 0;
    cut = false;
    for (int e = lane; e < entries; e += 32) {
        SeqShape s;
        int row0, rows;
        bool c;
        mine += entry_of(p, e, s, row0, rows, c);
        cut |= c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    return mine * p.kv.kv_heads;
}

// The unit that holds step `at` of the list (at < list_length), by a whole warp.
__device__ __forceinline__ ChunkUnit unit_at(const AttnParams &p, int64_t at, int lane)
{
    const int entries = p.kv.seqs * p.row_tiles;
    int64_t before = 0;
    ChunkUnit u;
    for (int e0 = 0;; e0 += 32) {
        int n = 0;
        if (e0 + lane < entries) {
            SeqShape s;
            int row0, rows;
            bool c;
            n = entry_of(p, e0 + lane, s, row0, rows, c);
        }
        int64_t upto = (int64_t)n * p.kv.kv_heads;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned hit = __ballot_sync(0xFFFFFFFFu, at < before + upto);
        if (hit) {
            const int l = __ffs(hit) - 1;
            u.e = e0 + l;
            bool c;
            u.steps = entry_of(p, u.e, u.s, u.row0, u.rows, c);
            const int64_t start = before + __shfl_sync(0xFFFFFFFFu, upto, l) - (int64_t)u.steps * p.kv.kv_heads;
            u.h = (int)((at - start) / u.steps);
            u.first = start + (int64_t)u.h * u.steps;
            return u;
        }
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
}

__device__ __forceinline__ void next_unit(const AttnParams &p, ChunkUnit &u)
{
    u.first += u.steps;
    if (++u.h < p.kv.kv_heads) return;
    u.h = 0;
    do {
        bool c;
        u.steps = entry_of(p, ++u.e, u.s, u.row0, u.rows, c);
    } while (u.steps == 0);
}

// One row's scores for kSpan tokens of a step as they came from tensor memory, times the keys' factors: u = 2^-b (q . K8),
// s = rc u; -infinity for tokens j0 .. that the row does not see (limit).
constexpr int kSpan = 32;
__device__ __forceinline__ void scores_of_row(uint32_t taddr, const float *factors, bool mask, int j0, int limit, f32x2 (&u)[kSpan / 2])
{
    uint32_t x[kSpan];
    tmem_load32(taddr, x);
    ulonglong2 f[kSpan / 4];                         // (the same address in all lanes; loaded while the scores are on their way)
#pragma unroll
    for (int k = 0; k < kSpan / 4; ++k) f[k] = reinterpret_cast<const ulonglong2 *>(factors)[k];
    tmem_wait_ld();
#pragma unroll
    for (int k = 0; k < kSpan / 2; k += 2) {
        const ulonglong2 f4 = f[k / 2];
        u[k] = mul2(pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), f4.x);
        u[k + 1] = mul2(pack2(__uint_as_float(x[2 * k + 2]), __uint_as_float(x[2 * k + 3])), f4.y);
    }
    if (__builtin_expect(mask, 0)) {
#pragma unroll
        for (int k = 0; k < kSpan / 2; ++k) {
            float lo, hi;
            unpack2(u[k], lo, hi);
            if (j0 + 2 * k >= limit) lo = -INFINITY;
            if (j0 + 2 * k + 1 >= limit) hi = -INFINITY;
            u[k] = pack2(lo, hi);
        }
    }
}

// u becomes the weights p = 2^(rc u - M); their sum.
__device__ __forceinline__ f32x2 weights_of_row(f32x2 (&u)[kSpan / 2], f32x2 rc2, float top)
{
    const f32x2 minus = pack2(-top, -top);
    f32x2 s[4];
#pragma unroll
    for (int k = 0; k < kSpan / 2; ++k) {
        float lo, hi;
        unpack2(fma2(u[k], rc2, minus), lo, hi);
        u[k] = pack2(exp2_approx(lo), exp2_approx(hi));
        s[k & 3] = k < 4 ? u[k] : add2(s[k & 3], u[k]);
    }
    return add2(add2(s[0], s[1]), add2(s[2], s[3]));
}

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 1) attn_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ AttnParams p)
{
    using L = ChunkShape<D>;
    constexpr int kFirstValueWarp = 8, kProductWarp = 12;
    extern __shared__ uint8_t smem_raw[];
    const KvParams &kv = p.kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // ---- the CTA's share of the list ----
    bool cut;
    const int64_t total = list_length(p, lane, cut);
    if (__builtin_expect(__any_sync(0xFFFFFFFFu, cut), 0)) {
        if (blockIdx.x == 0 && warp == 0 && lane == 0) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
        write_left_out_rows(kv, p.out, p.ld_o, p.lse, p.q_heads, D);
    }
    const int64_t share = max((total + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)p.min_share);
    const int64_t begin = blockIdx.x * share, end = min(total, begin + share);
    if (begin >= end) return;

    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem), bars = base + L::kBar;
    auto k_full = [&](uint32_t g) { return bars + 8u * (g % kKStages); };
    auto k_empty = [&](uint32_t g) { return bars + 8u * (kKStages + g % kKStages); };
    auto v_full = [&](uint32_t g) { return bars + 8u * (2 * kKStages + g % kVStages); };
    auto v_empty = [&](uint32_t g) { return bars + 8u * (2 * kKStages + kVStages + g % kVStages); };
    const uint32_t bars2 = bars + 8u * (2 * kKStages + 2 * kVStages);
    // of a slot's n-th step (four places each: the values' warps may be three steps ahead of a slot, and a slot that sits
    // out a unit must not meet a phase that it has not waited for)
    auto sc_full = [&](int q, uint32_t n) { return bars2 + 8u * (4 * q + (n & 3u)); };
    auto q_full = [&](int q) { return bars2 + 64u + 8u * q; };
    auto s_full = [&](int q) { return bars2 + 80u + 8u * q; };
    auto p_full = [&](int q) { return bars2 + 96u + 8u * q; };
    auto o_full = [&](int q) { return bars2 + 112u + 8u * q; };
    auto slot_bar = [&](int q) { return bars2 + 128u + 8u * q; };     // the 128 threads of a slot; both slots' 256
    const uint32_t both_bar = bars2 + 144u;
    auto pv_done = [&](int q) { return bars2 + 152u + 8u * q; };      // the slot's second product has read its weights
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::kBar + L::kNumBars * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    volatile int *is_last = reinterpret_cast<volatile int *>(tmem_slot + 2);     // [2]

    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kKStages; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); }
        for (uint32_t i = 0; i < kVStages; ++i) { mbar_init(v_full(i), 128); mbar_init(v_empty(i), 1); }
        for (int q = 0; q < 2; ++q) {
            for (uint32_t i = 0; i < 4; ++i) mbar_init(sc_full(q, i), 128);
            mbar_init(q_full(q), 128);
            mbar_init(s_full(q), 1);
            mbar_init(p_full(q), 4);
            mbar_init(o_full(q), 1);
            mbar_init(slot_bar(q), 128);
            mbar_init(pv_done(q), 1);
        }
        mbar_init(both_bar, 256);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kProductWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    const uint32_t tmem = *tmem_slot;

    ChunkUnit u = unit_at(p, begin, lane);
    int64_t at = begin;
    uint32_t g0 = 0;          // steps of this CTA before the current unit
    bool alive = true;

    if (warp == kProductWarp) {
        // ------------------------------- products -------------------------------
        const uint32_t idesc_s = (1u << 4) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);       // e4m3; a lo: e5m2
        const uint32_t idesc_o = (1u << 4) | (2u << 7) | (2u << 10) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);   // tf32
        uint32_t n_units[2] = {}, n_steps[2] = {}, n_scores[2] = {};
        const uint32_t tm = uniform(tmem), base_lo = uniform(desc_lo(base));
        auto wait = [&](uint32_t bar, uint32_t parity) {
            const bool ok = mbar_wait(bar, parity, abort_flag, kv.d_status);
            return (bool)__all_sync(0xFFFFFFFFu, ok);
        };
        // the weights in slot q's columns have been read (nothing to wait for before the slot's first scores: each of its
        // scores has one second product behind it)
        auto columns_free = [&](uint32_t q) {
            const uint32_t n = q ? n_scores[1]++ : n_scores[0]++;
            return n == 0 || wait(pv_done(q), (n - 1) & 1u);
        };
        // S of step g into slot q, from query tile qt
        auto scores = [&](uint32_t q, uint32_t qt, uint32_t g) {
            const uint32_t dk = base_lo + (L::kK + (g % kKStages) * L::kKBytes) / 16, dq = base_lo + (L::kQ + qt * L::kQBytes) / 16;
            if (elect_one()) {
#pragma unroll
                for (uint32_t term = 0; term < 2; ++term)
#pragma unroll
                    for (uint32_t k = 0; k < D / 32; ++k)
                        chunk_mma_f8<kSw128, D == 128 ? kSw128 : kSw64>(tm + kTmemSlot * q, dq + term * (D == 128 ? kTile * 128 / 16 : 4) + 2u * k,
                                                                        dk + 2u * k, idesc_s | term << 7, (term | k) ? 1u : 0u);
                chunk_commit(s_full(q));
            }
            __syncwarp();
        };
        // O of slot q += P of the slot, V of step g
        auto outputs = [&](uint32_t q, uint32_t g, uint32_t accumulate) {
            const uint32_t dv = base_lo + (L::kV + (g % kVStages) * L::kVBytes) / 16, slot = tm + kTmemSlot * q;
            if (elect_one()) {
#pragma unroll
                for (uint32_t k = 0; k < kTile / 8; ++k)      // eight tokens: 32 bytes of a block's rows, D * 128 bytes from block to block
                    chunk_mma_tf32_tmem<kSw128>(slot + kTmemO, slot + 8u * k, dv + (k >> 2) * (D * 128 / 16) + 2u * (k & 3), idesc_o,
                                                k == 0 ? accumulate : 1u);
                chunk_commit(pv_done(q));
            }
            __syncwarp();
        };
        auto commit = [&](uint32_t bar) {
            if (elect_one()) chunk_commit(bar);
            __syncwarp();
        };
        while (true) {
            const int lo = (int)(at - u.first);
            const int steps = (int)uniform((uint32_t)((int)min((int64_t)u.steps, end - u.first) - lo));
            const uint32_t two = uniform(u.rows > kTile);      // two query tiles; else even and odd steps
            g0 = uniform(g0);
            alive = wait(q_full(0), n_units[0]++ & 1u);
            if (two) alive = alive && wait(q_full(1), n_units[1]++ & 1u);
            alive = alive && wait(k_full(g0), (g0 / kKStages) & 1u) && columns_free(0);
            if (two) alive = alive && columns_free(1);
            if (!alive) break;
            chunk_fence_after();
            scores(0, 0, g0);
            if (two) scores(1, 1, g0);
            commit(k_empty(g0));
            if (!two && steps > 1) {
                alive = wait(k_full(g0 + 1), ((g0 + 1) / kKStages) & 1u) && columns_free(1);
                if (!alive) break;
                chunk_fence_after();
                scores(1, 0, g0 + 1);
                commit(k_empty(g0 + 1));
            }
            const int ahead = two ? 1 : 2;             // steps from one of a slot to its next
            for (int i = 0; i < steps; ++i) {
                const uint32_t g = g0 + i, gn = g + ahead;
                const bool last = i + ahead >= steps;
                if (!(alive = wait(v_full(g), (g / kVStages) & 1u))) break;
                const uint32_t q0 = two ? 0 : i & 1, q1 = two ? 1 : i & 1;
                for (uint32_t q = q0; q <= q1; ++q) {
                    if (!(alive = wait(p_full(q), (q ? n_steps[1]++ : n_steps[0]++) & 1u))) break;
                    chunk_fence_after();
                    outputs(q, g, i < ahead ? 0u : 1u);
                    if (q == q1) commit(v_empty(g));
                    if (last) {
                        commit(o_full(q));
                    } else {
                        if (q == q0) {
                            if (!(alive = wait(k_full(gn), (gn / kKStages) & 1u))) break;
                        }
                        if (!(alive = columns_free(q))) break;
                        chunk_fence_after();
                        scores(q, two ? q : 0, gn);
                        if (q == q1) commit(k_empty(gn));
                    }
                }
                if (!alive) break;
            }
            g0 += steps;
            at += steps;
            if (!alive || at >= end) break;
            next_unit(p, u);
        }
    } else if (warp >= kFirstValueWarp) {
        // ------------------------------- values, keys' loads, scaling biases -------------------------------
        // A warp takes 32 tokens of each tile, a lane one token's row: 32 lanes store one dimension of their tokens side
        // by side (all banks once).  Shared memory: four blocks of 32 tokens, [D][32 tokens], 128-byte rows, swizzled.
        const int cw = warp - kFirstValueWarp;
        constexpr int kLoads = D / 16;
        const int per_tile = kTile >> kv.page_shift, in_page = (1 << kv.page_shift) - 1;
        unsigned bad_pages = 0;
        uint32_t n_steps[2] = {}; // of the slots so far
        uint32_t place[8];        // of the lane's token in the rows of dimensions = 0 .. 7 mod 8
#pragma unroll
        for (int k = 0; k < 8; ++k) place[k] = base + L::kV + cw * (D * 128) + (((lane >> 2) ^ k) << 4) + ((lane & 3) << 2);
        while (true) {
            const int lo = (int)(at - u.first), steps = (int)min((int64_t)u.steps, end - u.first) - lo;
            const bool two = u.rows > kTile;
            const SeqShape s = u.s;
            const int32_t *table = kv.table + (int64_t)(u.e / p.row_tiles) * kv.table_stride;
            const int64_t row_h = (int64_t)u.h << kv.page_shift;
            const int last_page = s.len > 0 ? (s.len - 1) >> kv.page_shift : -1;
            // a token's page (-1: the token is behind the end, -2: the page number is out of range), its row and biases
            auto page_of_token = [&](int tile) {
                const int tk = tile * kTile + cw * 32 + lane;
                const int page = tk < s.len ? __ldg(table + (tk >> kv.page_shift)) : -1;
                return tk < s.len && (unsigned)page >= (unsigned)kv.pages ? -2 : page;
            };
            auto row_of = [&](int tile, int page, int &b_k, int &b_v) {
                const int64_t row = row_h + ((tile * kTile + cw * 32 + lane) & in_page);
                b_k = b_v = page == -1 ? 0 : FP8_KV_BIAS_NONFINITE;
                if (page == -2) bad_pages = 1;
                if (page < 0) return (const uint4 *)nullptr;
                b_k = kv.bk[page * kv.bias_stride + row];
                b_v = kv.bv[page * kv.bias_stride + row];
                return reinterpret_cast<const uint4 *>(kv.v8 + page * kv.page_stride + row * D);
            };
            uint4 cur[kLoads];
            int bk = 0, bv = 0, bk_n = 0, bv_n = 0, page_n = -1;
            // keys: the first of these warps, one lane per page of the tile
            auto page_of = [&](int tile) {
                const int j = tile * per_tile + lane;
                return lane < per_tile && j <= last_page ? __ldg(table + j) : 0;
            };
            auto request_keys = [&](int tile, uint32_t g, int page) {
                const bool load = lane < per_tile && tile * per_tile + lane <= last_page;
                const int n = __popc(__ballot_sync(0xFFFFFFFFu, load));
                const bool ok = mbar_wait(k_empty(g), ((g / kKStages) & 1u) ^ 1u, abort_flag, kv.d_status);
                if (!__all_sync(0xFFFFFFFFu, ok)) return false;
                if (lane == 0) mbar_expect_tx(k_full(g), (uint32_t)(n * D) << kv.page_shift);
                __syncwarp();
                // a page out of range is read as page 0; its tokens are marked non-finite below
                if (load)
                    tma_load_page(base + L::kK + (g % kKStages) * L::kKBytes + ((lane * D) << kv.page_shift), &map_k, k_full(g),
                                  u.h << kv.page_shift, (unsigned)page < (unsigned)kv.pages ? page : 0);
                __syncwarp();
                return true;
            };
            int page = 0;
            if (cw == 0) {
                alive = request_keys(lo, g0, page_of(lo));
                if (steps > 1) page = page_of(lo + 1);
            }
            {
                const uint4 *src = row_of(lo, page_of_token(lo), bk, bv);
#pragma unroll
                for (int k = 0; k < kLoads; ++k) cur[k] = src ? __ldg(src + k) : make_uint4(0, 0, 0, 0);
                if (steps > 1) page_n = page_of_token(lo + 1);
            }
            for (int i = 0; i < steps && alive; ++i) {
                const int tile = lo + i;
                const uint32_t g = g0 + i;
                // 2^-b of the key for the softmax (step g - 3 has used this place: its products, waited for a step ago, are done)
                const bool marked = bk == FP8_KV_BIAS_NONFINITE || bv == FP8_KV_BIAS_NONFINITE;
                reinterpret_cast<float *>(smem + L::kScale)[(g % 3u) * kTile + cw * 32 + lane] =
                    marked ? __int_as_float(0x7FFFFFFF) : key_factor(bk + kv.delta);
                const unsigned large = __ballot_sync(0xFFFFFFFFu, !marked && bv + kv.delta < kLargeValue);
                if (lane == 0) reinterpret_cast<unsigned *>(smem + L::kLarge)[(g % 3u) * 4 + cw] = large;
                if (two || (i & 1) == 0) mbar_arrive(sc_full(0, n_steps[0]++));
                if (two || (i & 1) == 1) mbar_arrive(sc_full(1, n_steps[1]++));
                if (cw == 0 && i + 1 < steps) {
                    alive = request_keys(tile + 1, g + 1, page);
                    if (!alive) break;
                    if (i + 2 < steps) page = page_of(tile + 2);
                }
                if (g >= 2) {         // the products of step g - 2 have read the values in this place
                    const bool ok = mbar_wait(v_empty(g), ((g / kVStages) & 1u) ^ 1u, abort_flag, kv.d_status);
                    if (!(alive = __all_sync(0xFFFFFFFFu, ok))) break;
                }
                // the next tile's row takes the registers as they are converted
                const uint4 *src_n = nullptr;
                if (i + 1 < steps) src_n = row_of(tile + 1, page_n, bk_n, bv_n);
                if (i + 2 < steps) page_n = page_of_token(tile + 2);
                const float f = pow2_normal(min(126, -(applied_bias(bv) + kv.delta)));
                const f32x2 f2 = pack2(f, f);
                const uint32_t stage = (g % kVStages) * L::kVBytes;
#pragma unroll
                for (int k = 0; k < kLoads; ++k) {
                    const uint32_t w[4] = {cur[k].x, cur[k].y, cur[k].z, cur[k].w};
                    cur[k] = src_n ? __ldg(src_n + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t h[2];
                        e4_to_f16(marked ? 0u : w[q], h[0], h[1]);     // (0 times a NaN byte would be one)
                        float v[4];
                        unpack4<FP8_F16>(h, v);
                        unpack2(mul2(pack2(v[0], v[1]), f2), v[0], v[1]);
                        unpack2(mul2(pack2(v[2], v[3]), f2), v[2], v[3]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int dim = 16 * k + 4 * q + j;
                            sts4(place[dim & 7] + stage + dim * 128, v[j]);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(v_full(g));
                bk = bk_n;
                bv = bv_n;
            }
            g0 += steps;
            at += steps;
            if (!alive || at >= end) break;
            next_unit(p, u);
        }
        if (bad_pages) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    } else {
        // ------------------------------- softmax and output -------------------------------
        const int slot = warp >> 2, r = threadIdx.x & 127;                     // slot, row of the query tile
        const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16, lanes = tmem + kTmemSlot * slot + quarter;
        uint32_t n_units[2] = {}, n_steps = 0, n_slot = 0, n_both = 0;      // units, steps, barriers so far
        // (barriers with a limit, like all waits: a warp that gave up does not leave the others waiting)
        auto sync_slot = [&]() {
            mbar_arrive(slot_bar(slot));
            const bool ok = mbar_wait(slot_bar(slot), n_slot++ & 1u, abort_flag, kv.d_status);
            return (bool)__all_sync(0xFFFFFFFFu, ok);
        };
        auto sync_both = [&]() {
            mbar_arrive(both_bar);
            const bool ok = mbar_wait(both_bar, n_both++ & 1u, abort_flag, kv.d_status);
            return (bool)__all_sync(0xFFFFFFFFu, ok);
        };
        while (true) {
            const int lo = (int)(at - u.first), hi = (int)min((int64_t)u.steps, end - u.first), steps = hi - lo;
            const SeqShape s = u.s;
            const bool two = u.rows > kTile, joined = !two && steps > 1;       // joined: the slots hold parts of one tile
            const int row0 = u.row0 + (two ? slot * kTile : 0), rows = u.rows - (two ? slot * kTile : 0);
            if (two || slot == 0 || joined) {
                const int tok = min((row0 + r) / p.group, s.n - 1), head = u.h * p.group + (row0 + r) % p.group;
                const int limit = tokens_seen(s, p.causal, (row0 + r) / p.group);   // tokens that the row sees
                // ---- queries as two 8-bit terms, one row per thread ----
                float rc;               // |c| / the row's power of two, and the keys' share
                {
                    const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (int64_t)(s.first + tok) * p.ld_q + (int64_t)head * D);
                    uint32_t m = 0;
                    if (r < rows) {
#pragma unroll 4
                        for (int i = 0; i < D / 8; ++i) {
                            const uint4 x = src[i];
                            m = max(m, max(max((x.x << 16) & 0x7FFF0000u, x.x & 0x7FFF0000u), max((x.y << 16) & 0x7FFF0000u, x.y & 0x7FFF0000u)));
                            m = max(m, max(max((x.z << 16) & 0x7FFF0000u, x.z & 0x7FFF0000u), max((x.w << 16) & 0x7FFF0000u, x.w & 0x7FFF0000u)));
                        }
                    }
                    unsigned ignored = 0;
                    const int e = min(126, bias_from_amax_bits(m, FP8_E4, FP8_CONV_NATIVE, 0, &ignored));   // the largest in (224, 448]
                    const float f = copysignf(pow2_normal(e), p.c);     // a negative scale goes into the queries: rc >= 0
                    // (not 0, and no NaN in a row that sees nothing: it multiplies the -infinity of masked tokens)
                    rc = m >= 0x7F800000u && limit > 0 ? __int_as_float(0x7FFFFFFF) : fmaxf(query_factor(fabsf(p.c), e), 1e-45f);
                    if (two || slot == 0) {
#pragma unroll 2
                        for (int i = 0; i < D / 16; ++i) {
                            uint4 x = make_uint4(0, 0, 0, 0), y = x;
                            if (r < rows) { x = src[2 * i]; y = src[2 * i + 1]; }
                            const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                            uint32_t hi4[4], lo4[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float a0 = __uint_as_float(w[2 * j] << 16) * f, a1 = __uint_as_float(w[2 * j] & 0xFFFF0000u) * f;
                                const float a2 = __uint_as_float(w[2 * j + 1] << 16) * f, a3 = __uint_as_float(w[2 * j + 1] & 0xFFFF0000u) * f;
                                hi4[j] = cvt_pair<FP8_E4>(a1, a0) | (cvt_pair<FP8_E4>(a3, a2) << 16);
                                uint32_t h2[2];
                                e4_to_f16(hi4[j], h2[0], h2[1]);
                                float back[4];
                                unpack4<FP8_F16>(h2, back);
                                lo4[j] = cvt_pair<FP8_E5>(a1 - back[1], a0 - back[0]) | (cvt_pair<FP8_E5>(a3 - back[3], a2 - back[2]) << 16);
                            }
                            // D = 128: a row of hi, and 16 KB on its row of lo; D = 64: hi and lo side by side in one 128-byte row
                            const int c_hi = i, c_lo = D == 128 ? i : i + 4;
                            const uint32_t row = base + L::kQ + slot * L::kQBytes + r * 128;
                            sts16(row + ((c_hi ^ (r & 7)) << 4), hi4[0], hi4[1], hi4[2], hi4[3]);
                            sts16(row + (D == 128 ? kTile * 128 : 0) + ((c_lo ^ (r & 7)) << 4), lo4[0], lo4[1], lo4[2], lo4[3]);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        mbar_arrive(q_full(slot));
                    }
                }
                const int least = __shfl_sync(0xFFFFFFFFu, limit, 0);   // the warp's first row sees least
                const bool active = (warp & 3) * 32 < rows;
                float top = kNoMax, sum_limit = kSumLimit;
                f32x2 sum = pack2(0.0f, 0.0f);
                const f32x2 rc2 = pack2(rc, rc);
                const int start = two ? 0 : slot, ahead = two ? 1 : 2;
                for (int i = start; i < steps; i += ahead) {
                    const uint32_t g = g0 + i;
                    const int t0 = (lo + i) * kTile;
                    bool ok = mbar_wait(sc_full(slot, n_steps), (n_steps >> 2) & 1u, abort_flag, kv.d_status);
                    ok = ok && mbar_wait(s_full(slot), n_steps & 1u, abort_flag, kv.d_status);
                    ++n_steps;
                    if (!(alive = __all_sync(0xFFFFFFFFu, ok))) break;
                    chunk_fence_after();
                    if (active) {
                        const float *factors = reinterpret_cast<const float *>(smem + L::kScale) + (g % 3u) * kTile;
                        const bool mask = t0 + kTile > least;
                        const uint4 large = *reinterpret_cast<const uint4 *>(smem + L::kLarge + (g % 3u) * 16);
                        if (large.x | large.y | large.z | large.w) sum_limit = kLargeSumLimit;
#pragma unroll 1
                        for (int c0 = 0; c0 < kTile; c0 += kSpan) {
                            f32x2 w[kSpan / 2];
                            scores_of_row(lanes + c0, factors + c0, mask, t0 + c0, limit, w);
                            // weights under M as it stands; only where their sum shows that a score lies far above M (or
                            // at the first token) is the maximum looked at, M moved and the weights taken again
                            f32x2 add = weights_of_row(w, rc2, top);
                            float a, b;
                            unpack2(add2(sum, add), a, b);
                            if (__builtin_expect(__any_sync(0xFFFFFFFFu, a + b > sum_limit), 0)) {
                                scores_of_row(lanes + c0, factors + c0, mask, t0 + c0, limit, w);
                                float m = -INFINITY;
#pragma unroll
                                for (int k = 0; k < kSpan / 2; ++k) {
                                    unpack2(w[k], a, b);
                                    m = fmaxf(m, fmaxf(a, b));
                                }
                                m = fmaf(m, rc, -kTf32Lift);
                                if (sum_limit != kSumLimit) {     // also above what the weights so far sum up to
                                    unpack2(sum, a, b);
                                    m = fmaxf(m, top + log2_approx(a + b)) + kLargeLift;
                                }
                                const float next = fmaxf(top, m), shrink = exp2_approx(top - next);
                                top = next;
                                sum = mul2(sum, pack2(shrink, shrink));
                                tmem_wait_st();
                                // this step's weights so far, and what has been summed before it
#pragma unroll 1
                                for (int k = 0; k < 8 + D / 16; ++k) {
                                    if (k < 8 ? 16 * k >= c0 : i == start) continue;
                                    uint32_t y[16];
                                    const uint32_t where = lanes + 16u * k;    // columns of P, then of O
                                    tmem_load16(where, y);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int q = 0; q < 16; ++q) y[q] = __float_as_uint(__uint_as_float(y[q]) * shrink);
                                    tmem_store16(where, y);
                                }
                                add = weights_of_row(w, rc2, top);
                            }
                            sum = add2(sum, add);
                            uint32_t y[kSpan];
#pragma unroll
                            for (int k = 0; k < kSpan / 2; ++k) {
                                unpack2(w[k], a, b);
                                y[2 * k] = __float_as_uint(a);
                                y[2 * k + 1] = __float_as_uint(b);
                            }
                            tmem_store32(lanes + c0, y);
                        }
                        tmem_wait_st();
                    }
                    chunk_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full(slot));
                }
                if (!alive) break;
                // ---- output: O of the slot, or of both slots under the larger M ----
                float l, scale0 = 1.0f, scale1 = 0.0f;
                {
                    float a, b;
                    unpack2(sum, a, b);
                    l = (a + b) * kTf32Kept;
                }
                bool ok = mbar_wait(o_full(slot), n_units[slot] & 1u, abort_flag, kv.d_status);
                float *stats = reinterpret_cast<float *>(smem + L::kQ + L::kQBytes);
                if (joined) {
                    if (slot == 0) ok = ok && mbar_wait(o_full(1), n_units[1] & 1u, abort_flag, kv.d_status);
                    else { stats[r] = top; stats[kTile + r] = l; }
                    if (!(alive = __all_sync(0xFFFFFFFFu, ok) && sync_both())) break;
                    if (slot == 0) {
                        const float top1 = stats[r], l1 = stats[kTile + r], both = fmaxf(top, top1);
                        scale0 = exp2_approx(top - both);
                        scale1 = exp2_approx(top1 - both);
                        l = l * scale0 + l1 * scale1;
                        top = both;
                    }
                } else if (!(alive = __all_sync(0xFFFFFFFFu, ok))) {
                    break;
                }
                chunk_fence_after();
                // 16 dimensions of the row's sum, from d on
                auto load_o = [&](int d, uint32_t (&y)[16]) {
                    tmem_load16(lanes + kTmemO + d, y);
                    if (joined) {
                        uint32_t z[16];
                        tmem_load16(lanes + kTmemSlot + kTmemO + d, z);
                        tmem_wait_ld();
#pragma unroll
                        for (int q = 0; q < 16; ++q) y[q] = __float_as_uint(fmaf(__uint_as_float(z[q]), scale1, __uint_as_float(y[q]) * scale0));
                    } else {
                        tmem_wait_ld();
                    }
                };
                const bool mine = r < rows;
                const int64_t out_row = s.first + tok;
                if (two || slot == 0) {
                    if (lo == 0 && hi == u.steps) {
                        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                        uint16_t *dst = p.out + out_row * p.ld_o + (int64_t)head * D;
                        if (active) {
#pragma unroll 2
                            for (int d = 0; d < D; d += 16) {
                                uint32_t x[16];
                                load_o(d, x);
                                uint32_t y[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q) y[q] = pack_bf16x2(__uint_as_float(x[2 * q]) * inv, __uint_as_float(x[2 * q + 1]) * inv);
                                if (mine) {
                                    *reinterpret_cast<uint4 *>(dst + d) = make_uint4(y[0], y[1], y[2], y[3]);
                                    *reinterpret_cast<uint4 *>(dst + d + 8) = make_uint4(y[4], y[5], y[6], y[7]);
                                }
                                __syncwarp();
                            }
                            if (mine && p.lse) p.lse[out_row * p.q_heads + head] = l == 0.0f ? -INFINITY : (top + log2_approx(l * (1.0f / kTf32Kept))) * kLn2;
                        }
                    } else {
                        // some of the unit's steps: sums and statistics to the workspace, joined in order by the last CTA
                        const int qt = two ? slot : 0;
                        const int64_t first_cta = u.first / share, last_cta = (u.first + u.steps - 1) / share;
                        float *part = p.part + (((int64_t)blockIdx.x * 2 + (lo == 0 ? 1 : 0)) * 2 + qt) * L::kPart;
                        if (active) {
#pragma unroll 2
                            for (int d = 0; d < D; d += 16) {
                                uint32_t x[16];
                                load_o(d, x);
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (mine) *reinterpret_cast<uint4 *>(part + r * D + d + 4 * k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                                __syncwarp();
                            }
                            if (mine) { part[kTile * D + r] = top; part[kTile * D + kTile + r] = l; }
                        }
                        __threadfence();
                        if (!(alive = sync_slot())) break;
                        if (r == 0) is_last[slot] = arrive(p.count + first_cta * 2 + qt, p.call) == (unsigned)(last_cta - first_cta);
                        if (!(alive = sync_slot())) break;
                        if (is_last[slot]) {
                            __threadfence();
                            if (r == 0) p.count[first_cta * 2 + qt] = 0ull;   // a captured call comes again under its number
                            // the first part lies in its CTA's place 1 (it starts at the unit's beginning), the others in place 0
                            auto part_of = [&](int64_t cta) { return p.part + ((cta * 2 + (cta == first_cta ? 1 : 0)) * 2 + qt) * L::kPart; };
                            constexpr int kPerRow = D / 4;           // lanes side by side along a row
                            // eight rows' loads at a time: their latency is what this costs
                            constexpr int kStep = 128 / kPerRow, kBatch = 8;
                            const int d = r % kPerRow * 4, most = min(rows, kTile);
                            for (int r0 = r / kPerRow; r0 < most; r0 += kBatch * kStep) {
                                JoinedRow joint[kBatch];
#pragma unroll
                                for (int k = 0; k < kBatch; ++k) join_start(joint[k]);
                                for (int64_t cta = first_cta; cta <= last_cta; ++cta) {
                                    const float *src = part_of(cta);
                                    float m[kBatch], l_part[kBatch];
                                    float4 y[kBatch];
#pragma unroll
                                    for (int k = 0; k < kBatch; ++k) {
                                        const int rr = min(r0 + k * kStep, most - 1);
                                        m[k] = __ldcg(src + kTile * D + rr);
                                        l_part[k] = __ldcg(src + kTile * D + kTile + rr);
                                        y[k] = __ldcg(reinterpret_cast<const float4 *>(src + rr * D + d));
                                    }
#pragma unroll
                                    for (int k = 0; k < kBatch; ++k) join_part(joint[k], m[k], l_part[k], y[k]);
                                }
#pragma unroll
                                for (int k = 0; k < kBatch; ++k) {
                                    const int rr = r0 + k * kStep;
                                    if (rr >= most) break;
                                    const JoinedRow &a = joint[k];
                                    const float inv = a.l == 0.0f ? 0.0f : 1.0f / a.l;
                                    const int64_t orow = s.first + (row0 + rr) / p.group;
                                    const int hd = u.h * p.group + (row0 + rr) % p.group;
                                    *reinterpret_cast<uint2 *>(p.out + orow * p.ld_o + (int64_t)hd * D + d) =
                                        make_uint2(pack_bf16x2(a.v.x * inv, a.v.y * inv), pack_bf16x2(a.v.z * inv, a.v.w * inv));
                                    if (p.lse && d == 0)
                                        p.lse[orow * p.q_heads + hd] = a.l == 0.0f ? -INFINITY : (a.m + log2_approx(a.l * (1.0f / kTf32Kept))) * kLn2;
                                }
                            }
                        }
                    }
                }
                if (joined) {         // the odd slot's sums have been read
                    chunk_fence_before();
                    if (!(alive = sync_both())) break;
                    chunk_fence_after();
                }
            }
            ++n_units[0];
            if (two || joined) ++n_units[1];
            g0 += steps;
            at += steps;
            if (at >= end) break;
            next_unit(p, u);
        }
    }

    // ------------------------------- teardown -------------------------------
    __syncwarp();
    if (*abort_flag) __nanosleep(20000);   // let copies and products already issued drain before the memory is released
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    if (warp == kProductWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// Map over the keys: [pages][kv_heads * page_size][D] bytes, one box = one head's tokens of one page.
static bool encode_keys(const fp8_ctx *ctx, CUtensorMap *map, const fp8_kv_cache_t *c)
{
    cuuint64_t dims[3] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->kv_heads * c->page_size, (cuuint64_t)c->pages};
    cuuint64_t strides[2] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->page_stride};
    cuuint32_t box[3] = {(cuuint32_t)c->head_dim, (cuuint32_t)c->page_size, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return ctx->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, c->k8, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                             c->head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t configure_attn_kernels()
{
    const cudaError_t e = cudaFuncSetAttribute(attn_chunk_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkShape<128>::kDynamic);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(attn_chunk_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkShape<64>::kDynamic);
}

template <int D>
static fp8_status_t launch_chunk(const fp8_ctx *ctx, AttnParams p, const fp8_kv_cache_t *c, cudaStream_t st)
{
    using L = ChunkShape<D>;
    const KvParams &kv = p.kv;
    const int64_t row_tiles = ((int64_t)kv.max_q_len * p.group + kUnitRows - 1) / kUnitRows;
    const int64_t units = row_tiles * kv.seqs * kv.kv_heads, longest = ((int64_t)kv.max_kv_len + kTile - 1) / kTile;
    if (row_tiles * kv.seqs > INT32_MAX) return FP8_ERR_SHAPE;
    p.row_tiles = (int)row_tiles;
    p.min_share = 4;      // steps: shorter shares spend more on starting and joining than they save
    int64_t grid = ctx->sm_count;
    const int64_t most = (units * longest + p.min_share - 1) / p.min_share;
    if (most < grid) grid = most;
    if (grid * 2 > kAttnCounters || grid * 4 * L::kPart * 4 > (int64_t)ctx->partial_bytes) return FP8_ERR_UNSUPPORTED;
    CUtensorMap map;
    if (!encode_keys(ctx, &map, c)) return FP8_ERR_CUDA;
    count_launch();
    attn_chunk_kernel<D><<<(unsigned)grid, kChunkThreads, L::kDynamic, st>>>(map, p);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

fp8_status_t attn_chunk(const fp8_ctx *ctx, const AttnParams &p, const fp8_kv_cache_t *c, cudaStream_t st)
{
    return c->head_dim == 128 ? launch_chunk<128>(ctx, p, c, st) : launch_chunk<64>(ctx, p, c, st);
}

}  // namespace fp8lin
