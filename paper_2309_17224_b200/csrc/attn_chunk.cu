// Attention over the paged FP8 cache for many query rows: chunks of a prompt, drafted tokens.
//
// The query rows of one key/value head (token by token, the head's query heads side by side) are taken in tiles of 128,
// NQ tiles to a CTA, and the cached tokens in tiles of 128; two products per pair of tiles on the 5th-generation tensor
// cores:
//   S = Q K^T   e4m3 x e4m3: the cache's key bytes are the operand as they lie (TMA, no conversion).  A query row is the
//               sum of two e4m3 numbers under one power of two, q 2^e = hi + lo (hi rounded to nearest, lo the rest):
//               eight significant bits together, so bf16 queries are exact unless 2^17 below their row's largest.  Two
//               e4m3 products cost what one bf16 product costs.
//   O += P V    bf16: a value 2^-d V8 is a bf16 number; four warps make them on their way into shared memory (once for
//               all query rows of the CTA).  P in its two bf16 terms is read from tensor memory, where it takes the place
//               of the scores that it came from, 32 tokens' terms side by side.
// So a pair of tiles costs the tensor cores three bf16 products where bf16 attention has two.
//
// NQ = 2 (more than 128 rows): one CTA per SM, all 512 tensor-memory columns; while one tile's softmax runs, the other's
// products do, and the values are converted once for 256 rows.  NQ = 1 (up to 128 rows): two CTAs per SM do the same for
// one another.  Within a tile the order is strict: S, softmax, O, next S; that also makes the rescaling of O safe without
// a barrier of its own, as S of a step is complete only after O of the step before.
//
// The steps (tiles of tokens) of all units (query tiles of a key/value head) form one list that is cut evenly between the
// CTAs, whatever the sequences' lengths and the mask; a unit that lies in several CTAs leaves partial sums in the
// workspace, joined in order by the CTA that arrives last.
//
// Warps: 0 .. 4 NQ - 1 softmax and output (one query row per thread), then four for values, key loads and scaling
// biases, one for the products.
#include "attn_common.cuh"
#include "ptx.cuh"

namespace fp8lin {

constexpr int kTile = 128;                 // query rows of a tile, and tokens of a step
constexpr int kKStages = 2;

template <int D, int NQ>
struct ChunkShape {
    static constexpr int kThreads = 32 * (4 * NQ + 5);
    static constexpr int kResident = NQ == 1 ? 2 : 1;        // CTAs per SM
    static constexpr int kVStages = NQ == 1 ? 1 : 2;
    static constexpr int kQBytes = kTile * 2 * D;            // of one query tile
    static constexpr int kKBytes = kTile * D;
    static constexpr int kVBytes = kTile * D * 2;
    static constexpr int kQ = 0;
    static constexpr int kK = kQ + NQ * kQBytes;
    static constexpr int kV = kK + kKStages * kKBytes;
    static constexpr int kScale = kV + kVStages * kVBytes;   // [2][128] floats: 2^-b of a tile's keys
    static constexpr int kBar = kScale + 2 * kTile * 4;
    static constexpr int kNumBars = 2 * kKStages + 2 * kVStages + 2 + 4 * NQ;
    static constexpr int kTotal = kBar + kNumBars * 8 + 16;
    static constexpr int kDynamic = kTotal + 1024;           // slack to align the base to 1024 bytes
    static constexpr uint32_t kTmemCols = 256 * NQ;          // per query tile 128 columns of S, then P; 128 of O
    static constexpr int kPart = kTile * (D + 2);            // floats of a tile's partial result: sums, M, denominators
};
constexpr uint32_t kTmemO = 128;

__device__ __forceinline__ void chunk_mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
                 "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void chunk_mma_bf16_tmem(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
                 "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
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
// Two pairs of floats from shared memory (the same address in all lanes: one wavefront).
__device__ __forceinline__ void lds_pairs(uint32_t addr, f32x2 &a, f32x2 &b)
{
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(addr));
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Shared-memory matrix descriptors (start address, leading and stride offsets in 16-byte units, version 1, swizzle).
//   128-byte swizzle, operand rows of 128 contiguous bytes along the contraction, groups of eight rows 1024 bytes apart
//   64-byte swizzle, rows of 64 bytes, groups of eight rows 512 bytes apart
//   128-byte swizzle, contraction rows of 128 bytes of the N index, eight of them 1024 bytes; N blocks `lbo` apart
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr, uint32_t lbo)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t desc_sw64(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (uint64_t)1 << 16 | (uint64_t)(512 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)4 << 61;
}

__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap *map, uint32_t bar, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(y), "r"(z)
                 : "memory");
}

// A unit of the list: NQ query tiles of one key/value head.
struct ChunkUnit {
    int e;            // entry: sequence * row_tiles + place of the tiles in the sequence
    int h;
    SeqShape s;
    int row0, rows;   // first row, rows from there on
    int steps;        // tiles of tokens that any of the unit's rows sees (at least one)
    int64_t first;    // place of the unit's first step in the list
};

template <int NQ>
__device__ __forceinline__ int entry_of(const AttnParams &p, int e, SeqShape &s, int &row0, int &rows, bool &cut)
{
    const int b = e / p.row_tiles;
    s = seq_shape(p.kv, b, cut);
    row0 = (e - b * p.row_tiles) * (NQ * kTile);
    rows = (int)min((int64_t)s.n * p.group - row0, (int64_t)(NQ * kTile));
    if (rows <= 0) return 0;
    int see = s.len;
    if (p.causal) see = min(s.len, max(0, s.len - s.n + (row0 + rows - 1) / p.group + 1));
    return max(1, (see + kTile - 1) / kTile);
}

// Length of the list, by a whole warp.
template <int NQ>
__device__ __forceinline__ int64_t list_length(const AttnParams &p, int lane, bool &cut)
{
    const int entries = p.kv.seqs * p.row_tiles;
    int64_t mine = 0;
    cut = false;
    for (int e = lane; e < entries; e += 32) {
        SeqShape s;
        int row0, rows;
        bool c;
        mine += entry_of<NQ>(p, e, s, row0, rows, c);
        cut |= c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    return mine * p.kv.kv_heads;
}

// The unit that holds step `at` of the list (at < list_length), by a whole warp.
template <int NQ>
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
            n = entry_of<NQ>(p, e0 + lane, s, row0, rows, c);
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
            u.steps = entry_of<NQ>(p, u.e, u.s, u.row0, u.rows, c);
            const int64_t start = before + __shfl_sync(0xFFFFFFFFu, upto, l) - (int64_t)u.steps * p.kv.kv_heads;
            u.h = (int)((at - start) / u.steps);
            u.first = start + (int64_t)u.h * u.steps;
            return u;
        }
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
}

template <int NQ>
__device__ __forceinline__ void next_unit(const AttnParams &p, ChunkUnit &u)
{
    u.first += u.steps;
    if (++u.h < p.kv.kv_heads) return;
    u.h = 0;
    do {
        bool c;
        u.steps = entry_of<NQ>(p, ++u.e, u.s, u.row0, u.rows, c);
    } while (u.steps == 0);
}

// The weights of 32 tokens for one row: p = 2^(rc u - M) in two bf16 terms, and their sum.
__device__ __forceinline__ f32x2 weights32(const f32x2 (&u)[16], f32x2 rc2, float top, uint32_t (&ph)[32])
{
    const f32x2 minus = pack2(-top, -top);
    f32x2 s0 = pack2(0.0f, 0.0f), s1 = s0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        float lo, hi;
        unpack2(fma2(u[k], rc2, minus), lo, hi);
        lo = exp2_approx(lo);
        hi = exp2_approx(hi);
        const f32x2 both = pack2(lo, hi);
        if (k & 1) s1 = add2(s1, both);
        else s0 = add2(s0, both);
        const uint32_t a = __float_as_uint(lo), b = __float_as_uint(hi);
        ph[k] = __byte_perm(a, b, 0x7632);                       // the leading eight bits ...
        const f32x2 rest = add2(both, pack2(__uint_as_float((a & 0xFFFF0000u) ^ 0x80000000u), __uint_as_float((b & 0xFFFF0000u) ^ 0x80000000u)));
        unpack2(rest, lo, hi);
        ph[16 + k] = pack_bf16x2(lo, hi);                        // ... and what they leave
    }
    return add2(s0, s1);
}

template <int D, int NQ>
__global__ void __launch_bounds__((ChunkShape<D, NQ>::kThreads), (ChunkShape<D, NQ>::kResident))
attn_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const AttnParams p)
{
    using L = ChunkShape<D, NQ>;
    constexpr int kVS = L::kVStages;
    constexpr int kFirstValueWarp = 4 * NQ, kProductWarp = 4 * NQ + 4;
    extern __shared__ uint8_t smem_raw[];
    const KvParams &kv = p.kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // ---- the CTA's share of the list ----
    bool cut;
    const int64_t total = list_length<NQ>(p, lane, cut);
    if (blockIdx.x == 0 && warp == 0 && __any_sync(0xFFFFFFFFu, cut) && lane == 0) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    const int64_t share = max((total + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)p.min_share);
    const int64_t begin = blockIdx.x * share, end = min(total, begin + share);
    if (begin >= end) return;

    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem), bars = base + L::kBar;
    auto k_full = [&](uint32_t g) { return bars + 8u * (g % kKStages); };
    auto k_empty = [&](uint32_t g) { return bars + 8u * (kKStages + g % kKStages); };
    auto v_full = [&](uint32_t g) { return bars + 8u * (2 * kKStages + g % kVS); };
    auto v_empty = [&](uint32_t g) { return bars + 8u * (2 * kKStages + kVS + g % kVS); };
    const uint32_t bars2 = bars + 8u * (2 * kKStages + 2 * kVS);
    auto sc_full = [&](uint32_t g) { return bars2 + 8u * (g & 1u); };
    auto q_full = [&](int q) { return bars2 + 16u + 8u * q; };
    auto s_full = [&](int q) { return bars2 + 16u + 8u * (NQ + q); };
    auto p_full = [&](int q) { return bars2 + 16u + 8u * (2 * NQ + q); };
    auto o_full = [&](int q) { return bars2 + 16u + 8u * (3 * NQ + q); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::kBar + L::kNumBars * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    volatile int *is_last = reinterpret_cast<volatile int *>(tmem_slot + 2);     // [NQ]

    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kKStages; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); }
        for (uint32_t i = 0; i < kVS; ++i) { mbar_init(v_full(i), 128); mbar_init(v_empty(i), 1); }
        for (uint32_t i = 0; i < 2; ++i) mbar_init(sc_full(i), 128);
        for (int q = 0; q < NQ; ++q) {
            mbar_init(q_full(q), 128);
            mbar_init(s_full(q), 1);
            mbar_init(p_full(q), 4);
            mbar_init(o_full(q), 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kProductWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(L::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    const uint32_t tmem = *tmem_slot;

    ChunkUnit u = unit_at<NQ>(p, begin, lane);
    int64_t at = begin;
    uint32_t g0 = 0;          // steps of this CTA before the current unit
    bool alive = true;

    if (warp == kProductWarp) {
        // ------------------------------- products -------------------------------
        const uint32_t idesc_s = (1u << 4) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);   // e4m3 x e4m3
        const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) |
                                 ((uint32_t)(kTile >> 4) << 24);                                                 // bf16, B along N
        uint32_t n_units[NQ] = {}, n_steps[NQ] = {};
        auto scores = [&](int q, uint32_t g) {
            const uint32_t k_addr = base + L::kK + (g % kKStages) * L::kKBytes, q_addr = base + L::kQ + q * L::kQBytes;
            const uint64_t dk = D == 128 ? desc_sw128(k_addr, 16) : desc_sw64(k_addr);
#pragma unroll
            for (int term = 0; term < 2; ++term) {
                const uint64_t dq = D == 128 ? desc_sw128(q_addr + term * kTile * 128, 16) : desc_sw128(q_addr, 16) + 4u * term;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) chunk_mma_f8(tmem + 256u * q, dq + 2u * k, dk + 2u * k, idesc_s, (term | k) ? 1u : 0u);
            }
        };
        if (lane == 0) {
            while (true) {
                const int lo = (int)(at - u.first), steps = (int)min((int64_t)u.steps, end - u.first) - lo;
                const int nq = NQ == 1 || u.rows <= kTile ? 1 : 2;
                for (int q = 0; q < nq && alive; ++q) alive = mbar_wait(q_full(q), n_units[q]++ & 1u, abort_flag, kv.d_status);
                alive = alive && mbar_wait(k_full(g0), (g0 / kKStages) & 1u, abort_flag, kv.d_status);
                if (!alive) break;
                chunk_fence_after();
                for (int q = 0; q < nq; ++q) {
                    scores(q, g0);
                    chunk_commit(s_full(q));
                }
                chunk_commit(k_empty(g0));
                for (int i = 0; i < steps && alive; ++i) {
                    const uint32_t g = g0 + i;
                    const uint64_t dv = desc_sw128(base + L::kV + (g % kVS) * L::kVBytes, kTile * 128);
                    alive = mbar_wait(v_full(g), (g / kVS) & 1u, abort_flag, kv.d_status);
                    for (int q = 0; q < nq && alive; ++q) {
                        alive = mbar_wait(p_full(q), n_steps[q]++ & 1u, abort_flag, kv.d_status);
                        if (!alive) break;
                        chunk_fence_after();
                        const uint32_t acc = tmem + 256u * q + kTmemO;
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k) {      // 16 tokens: columns 8 (k % 2) of the 32 that hold 32 tokens
                            const uint32_t p1 = tmem + 256u * q + 32u * (k >> 1) + 8u * (k & 1);
                            chunk_mma_bf16_tmem(acc, p1, dv + 128u * k, idesc_o, (i | k) ? 1u : 0u);
                            chunk_mma_bf16_tmem(acc, p1 + 16u, dv + 128u * k, idesc_o, 1u);
                        }
                        if (q == nq - 1) chunk_commit(v_empty(g));
                        if (i + 1 == steps) {
                            chunk_commit(o_full(q));
                        } else {
                            if (q == 0) {
                                alive = mbar_wait(k_full(g + 1), ((g + 1) / kKStages) & 1u, abort_flag, kv.d_status);
                                if (!alive) break;
                                chunk_fence_after();
                            }
                            scores(q, g + 1);
                            chunk_commit(s_full(q));
                            if (q == nq - 1) chunk_commit(k_empty(g + 1));
                        }
                    }
                }
                g0 += steps;
                at += steps;
                if (!alive || at >= end) break;
                next_unit<NQ>(p, u);
            }
        }
    } else if (warp >= kFirstValueWarp) {
        // ------------------------------- values, keys' loads, scaling biases -------------------------------
        // A warp takes 32 tokens of each tile: lane (tok, c) = (lane / 4, lane % 4) of eight tokens at a time, 16 bytes.
        // Two neighbouring tokens and four pieces of 16 dimensions meet all banks once in each store of eight lanes.
        const int cw = warp - kFirstValueWarp, sub = lane >> 2, c = lane & 3;
        constexpr int kHalves = D / 64, kLoads = 4 * kHalves;
        const int per_tile = kTile >> kv.page_shift, in_page = (1 << kv.page_shift) - 1;
        unsigned bad_pages = 0;
        while (true) {
            const int lo = (int)(at - u.first), steps = (int)min((int64_t)u.steps, end - u.first) - lo;
            const SeqShape s = u.s;
            const int32_t *table = kv.table + (int64_t)(u.e / p.row_tiles) * kv.table_stride;
            const int64_t row_h = (int64_t)u.h << kv.page_shift;
            const int last_page = s.len > 0 ? (s.len - 1) >> kv.page_shift : -1;
            uint4 cur[kLoads], nxt[kLoads];
            int bk = 0, bv = 0, bk_n = 0, bv_n = 0;
            auto request = [&](int tile, uint4 (&v)[kLoads], int &b_k, int &b_v) {
                // pages of the warp's tokens 0..15 and 16..31 (the same one unless pages hold 16 tokens)
                const int t0 = tile * kTile + cw * 32;
                int pg[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    pg[i] = t0 + 16 * i < s.len ? __ldg(table + ((t0 + 16 * i) >> kv.page_shift)) : 0;
                    if ((unsigned)pg[i] >= (unsigned)kv.pages) { pg[i] = -1; bad_pages = 1; }
                }
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int g8 = i / kHalves, half = i % kHalves;           // eight tokens g8 * 8 + sub
                    const int tk = t0 + g8 * 8 + sub;
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (tk < s.len && pg[g8 >> 1] >= 0)
                        v[i] = ldg_stream(kv.v8 + pg[g8 >> 1] * kv.page_stride + (row_h + (tk & in_page)) * D + half * 64 + c * 16);
                }
                const int tk = t0 + lane, mine = lane < 16 ? pg[0] : pg[1];
                b_k = b_v = 0;
                if (tk < s.len) {
                    b_k = b_v = FP8_KV_BIAS_NONFINITE;
                    if (mine >= 0) {
                        const int64_t where = mine * kv.bias_stride + row_h + (tk & in_page);
                        b_k = kv.bk[where];
                        b_v = kv.bv[where];
                    }
                }
            };
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
            if (alive) request(lo, cur, bk, bv);
            for (int i = 0; i < steps && alive; ++i) {
                const int tile = lo + i;
                const uint32_t g = g0 + i;
                if (cw == 0 && i + 1 < steps) {
                    alive = request_keys(tile + 1, g + 1, page);
                    if (!alive) break;
                    if (i + 2 < steps) page = page_of(tile + 2);
                }
                auto wait_free = [&](uint32_t gg) {        // the products of step gg have read their values
                    const bool ok = mbar_wait(v_empty(gg), (gg / kVS) & 1u, abort_flag, kv.d_status);
                    return (bool)__all_sync(0xFFFFFFFFu, ok);
                };
                if (kVS == 2 && g >= 2 && !(alive = wait_free(g - 2))) break;
                // the tile's factors: 2^-b of the keys for the softmax (its reader two steps ago is done: the products
                // of that step, waited for above or a step ago, followed it), 2^(120 - d) for the values
                const bool marked = bk == FP8_KV_BIAS_NONFINITE || bv == FP8_KV_BIAS_NONFINITE;
                const unsigned drop = __ballot_sync(0xFFFFFFFFu, marked);
                reinterpret_cast<float *>(smem + L::kScale)[(g & 1u) * kTile + cw * 32 + lane] =
                    marked ? __int_as_float(0x7FFFFFFF) : pow2_normal(min(126, -(bk + kv.delta)));
                const uint32_t factor = value_factor(bv + kv.delta), rest = value_factor_rest(bv + kv.delta);
                const bool two_steps = __any_sync(0xFFFFFFFFu, bv + kv.delta < -7);     // values beyond 2^15
                mbar_arrive(sc_full(g));
                if (i + 1 < steps) request(tile + 1, nxt, bk_n, bv_n);
                if (kVS == 1 && g >= 1 && !(alive = wait_free(g - 1))) break;
#pragma unroll
                for (int k = 0; k < kLoads; ++k) {
                    const int g8 = k / kHalves, half = k % kHalves, tk = cw * 32 + g8 * 8 + sub;
                    uint4 v = cur[k];
                    if ((drop >> (g8 * 8 + sub)) & 1u) v = make_uint4(0, 0, 0, 0);   // 0 times a NaN byte would be one
                    const uint32_t f = __shfl_sync(0xFFFFFFFFu, factor, g8 * 8 + sub) * 0x10001u;
                    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
                    uint32_t w[8];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        w[2 * q] = mul_bf16x2(e4_fields_as_bf16(__byte_perm(x[q], 0u, 0x1000)), f);
                        w[2 * q + 1] = mul_bf16x2(e4_fields_as_bf16(__byte_perm(x[q], 0u, 0x3020)), f);
                    }
                    if (two_steps) {
                        const uint32_t f2 = __shfl_sync(0xFFFFFFFFu, rest, g8 * 8 + sub) * 0x10001u;
#pragma unroll
                        for (int q = 0; q < 8; ++q) w[q] = mul_bf16x2(w[q], f2);
                    }
                    const uint32_t row = base + L::kV + (g % kVS) * L::kVBytes + half * (kTile * 128) + tk * 128;
                    sts16(row + (((2 * c) ^ (tk & 7)) << 4), w[0], w[1], w[2], w[3]);
                    sts16(row + (((2 * c + 1) ^ (tk & 7)) << 4), w[4], w[5], w[6], w[7]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(v_full(g));
#pragma unroll
                for (int k = 0; k < kLoads; ++k) cur[k] = nxt[k];
                bk = bk_n;
                bv = bv_n;
            }
            g0 += steps;
            at += steps;
            if (!alive || at >= end) break;
            next_unit<NQ>(p, u);
        }
        if (bad_pages) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    } else {
        // ------------------------------- softmax and output -------------------------------
        const int qt = NQ == 1 ? 0 : warp >> 2, r = threadIdx.x & 127;         // query tile, row in it
        const uint32_t lanes = tmem + 256u * qt + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t n_units = 0, n_steps = 0;
        while (true) {
            const int lo = (int)(at - u.first), hi = (int)min((int64_t)u.steps, end - u.first), steps = hi - lo;
            const SeqShape s = u.s;
            const int row0 = u.row0 + qt * kTile, rows = u.rows - qt * kTile;  // of this query tile
            if (rows > 0) {
                const int tok = min((row0 + r) / p.group, s.n - 1), head = u.h * p.group + (row0 + r) % p.group;
                // ---- queries as two e4m3 terms, one row per thread ----
                float rc;               // |c| / the row's power of two
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
                    // (not 0: it multiplies the -infinity of masked tokens)
                    rc = m >= 0x7F800000u ? __int_as_float(0x7FFFFFFF) : fmaxf(fabsf(p.c) * pow2_normal(-e), 1e-37f);
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
                            lo4[j] = cvt_pair<FP8_E4>(a1 - back[1], a0 - back[0]) | (cvt_pair<FP8_E4>(a3 - back[3], a2 - back[2]) << 16);
                        }
                        // D = 128: a row of hi, and 16 KB on its row of lo; D = 64: hi and lo side by side in one 128-byte row
                        const int c_hi = i, c_lo = D == 128 ? i : i + 4;
                        const uint32_t row = base + L::kQ + qt * L::kQBytes + r * 128;
                        sts16(row + ((c_hi ^ (r & 7)) << 4), hi4[0], hi4[1], hi4[2], hi4[3]);
                        sts16(row + (D == 128 ? kTile * 128 : 0) + ((c_lo ^ (r & 7)) << 4), lo4[0], lo4[1], lo4[2], lo4[3]);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    mbar_arrive(q_full(qt));
                }
                int limit = s.len;       // tokens that the row sees
                if (p.causal) limit = min(s.len, max(0, s.len - s.n + (row0 + r) / p.group + 1));
                const int least = __shfl_sync(0xFFFFFFFFu, limit, 0);   // the warp's first row sees least
                const bool active = (warp & 3) * 32 < rows;
                float top = kNoMax;
                f32x2 sum = pack2(0.0f, 0.0f);
                const f32x2 rc2 = pack2(rc, rc);
                for (int i = 0; i < steps; ++i) {
                    const uint32_t g = g0 + i;
                    const int t0 = (lo + i) * kTile;
                    bool ok = mbar_wait(s_full(qt), n_steps++ & 1u, abort_flag, kv.d_status);
                    ok = ok && mbar_wait(sc_full(g), (g >> 1) & 1u, abort_flag, kv.d_status);
                    if (!(alive = __all_sync(0xFFFFFFFFu, ok))) break;
                    chunk_fence_after();
                    if (active) {
                        const uint32_t sc = base + L::kScale + (g & 1u) * (kTile * 4);
                        const bool mask = t0 + kTile > least;
#pragma unroll 1
                        for (int ch = 0; ch < 4; ++ch) {
                            uint32_t x[32];
                            tmem_load32(lanes + 32u * ch, x);
                            tmem_wait_ld();
                            // v = 2^-b (q . K8), s = rc v
                            f32x2 v[16];
#pragma unroll
                            for (int k = 0; k < 16; k += 2) {
                                f32x2 f0, f1;
                                lds_pairs(sc + (ch * 32 + 2 * k) * 4, f0, f1);
                                v[k] = mul2(pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), f0);
                                v[k + 1] = mul2(pack2(__uint_as_float(x[2 * k + 2]), __uint_as_float(x[2 * k + 3])), f1);
                            }
                            if (mask) {
#pragma unroll
                                for (int k = 0; k < 16; ++k) {
                                    float a, b;
                                    unpack2(v[k], a, b);
                                    const int j = t0 + ch * 32 + 2 * k;
                                    if (j >= limit) a = -INFINITY;
                                    if (j + 1 >= limit) b = -INFINITY;
                                    v[k] = pack2(a, b);
                                }
                            }
                            // weights under M as it stands; only where their sum shows that a score lies far above M (or
                            // at the first token) is the maximum looked at, M moved and the weights taken again
                            uint32_t ph[32];
                            f32x2 add = weights32(v, rc2, top, ph);
                            float a, b;
                            unpack2(add2(sum, add), a, b);
                            if (__any_sync(0xFFFFFFFFu, a + b > kSumLimit)) {
                                float m = -INFINITY;
#pragma unroll
                                for (int k = 0; k < 16; ++k) {
                                    unpack2(v[k], a, b);
                                    m = fmaxf(m, fmaxf(a, b));
                                }
                                m *= rc;
                                // by a whole number of powers of two: exact for the bf16 weights already written
                                const float next = m > top ? (top == kNoMax ? m : top + ceilf(m - top)) : top, shrink = exp2_approx(top - next);
                                top = next;
                                sum = mul2(sum, pack2(shrink, shrink));
                                tmem_wait_st();
                                const uint32_t shrink_h = pack_bf16x2(shrink, shrink);
                                for (int k = 0; k < 2 * ch; ++k) {
                                    uint32_t y[16];
                                    tmem_load16(lanes + 16u * k, y);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int q = 0; q < 16; ++q) y[q] = mul_bf16x2(y[q], shrink_h);
                                    tmem_store16(lanes + 16u * k, y);
                                }
                                if (i > 0) {
                                    for (int k = 0; k < D / 16; ++k) {
                                        uint32_t y[16];
                                        tmem_load16(lanes + kTmemO + 16u * k, y);
                                        tmem_wait_ld();
#pragma unroll
                                        for (int q = 0; q < 16; ++q) y[q] = __float_as_uint(__uint_as_float(y[q]) * shrink);
                                        tmem_store16(lanes + kTmemO + 16u * k, y);
                                    }
                                }
                                add = weights32(v, rc2, top, ph);
                            }
                            sum = add2(sum, add);
                            tmem_store32(lanes + 32u * ch, ph);
                        }
                        tmem_wait_st();
                    }
                    chunk_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full(qt));
                }
                if (!alive) break;
                // ---- output ----
                float l;
                {
                    float a, b;
                    unpack2(sum, a, b);
                    l = a + b;
                }
                const bool ok = mbar_wait(o_full(qt), n_units++ & 1u, abort_flag, kv.d_status);
                if (!(alive = __all_sync(0xFFFFFFFFu, ok))) break;
                chunk_fence_after();
                const bool mine = r < rows;
                const int64_t out_row = s.first + tok;
                if (lo == 0 && hi == u.steps) {
                    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                    uint16_t *dst = p.out + out_row * p.ld_o + (int64_t)head * D;
                    if (active) {
#pragma unroll 1
                        for (int ch = 0; ch < D / 32; ++ch) {
                            uint32_t x[32];
                            tmem_load32(lanes + kTmemO + 32u * ch, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                uint32_t y[4];
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    y[q] = pack_bf16x2(__uint_as_float(x[8 * k + 2 * q]) * inv, __uint_as_float(x[8 * k + 2 * q + 1]) * inv);
                                if (mine) *reinterpret_cast<uint4 *>(dst + ch * 32 + k * 8) = make_uint4(y[0], y[1], y[2], y[3]);
                            }
                            __syncwarp();
                        }
                        if (mine && p.lse) p.lse[out_row * p.q_heads + head] = l == 0.0f ? -INFINITY : (top + log2_approx(l)) * kLn2;
                    }
                } else {
                    // some of the unit's steps: sums and statistics to the workspace, joined in order by the last CTA
                    const int64_t first_cta = u.first / share, last_cta = (u.first + u.steps - 1) / share;
                    float *slot = p.part + (((int64_t)blockIdx.x * 2 + (lo == 0 ? 1 : 0)) * NQ + qt) * L::kPart;
                    if (active) {
#pragma unroll 1
                        for (int ch = 0; ch < D / 32; ++ch) {
                            uint32_t x[32];
                            tmem_load32(lanes + kTmemO + 32u * ch, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (mine) *reinterpret_cast<uint4 *>(slot + r * D + ch * 32 + 4 * k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                            __syncwarp();
                        }
                        if (mine) { slot[kTile * D + r] = top; slot[kTile * D + kTile + r] = l; }
                    }
                    __threadfence();
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + qt) : "memory");
                    if (r == 0) is_last[qt] = atomicAdd(p.count + first_cta * NQ + qt, 1u) == (unsigned)(last_cta - first_cta);
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + qt) : "memory");
                    if (is_last[qt]) {
                        __threadfence();
                        if (r == 0) p.count[first_cta * NQ + qt] = 0u;
                        // the first part lies in its CTA's slot 1 (it starts at the unit's beginning), the others in slot 0
                        auto part_of = [&](int64_t cta) { return p.part + ((cta * 2 + (cta == first_cta ? 1 : 0)) * NQ + qt) * L::kPart; };
                        constexpr int kPerRow = D / 4;           // lanes side by side along a row
                        for (int rr = r / kPerRow; rr < min(rows, kTile); rr += 128 / kPerRow) {
                            const int d = r % kPerRow * 4;
                            float m = kNoMax;
                            for (int64_t k = first_cta; k <= last_cta; ++k) m = fmaxf(m, __ldcg(part_of(k) + kTile * D + rr));
                            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                            float sum_l = 0.0f;
                            for (int64_t k = first_cta; k <= last_cta; ++k) {
                                const float *src = part_of(k);
                                const float f = exp2_approx(__ldcg(src + kTile * D + rr) - m);
                                const float4 y = __ldcg(reinterpret_cast<const float4 *>(src + rr * D + d));
                                v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
                                sum_l = fmaf(__ldcg(src + kTile * D + kTile + rr), f, sum_l);
                            }
                            const float inv = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;
                            const int64_t orow = s.first + (row0 + rr) / p.group;
                            const int hd = u.h * p.group + (row0 + rr) % p.group;
                            *reinterpret_cast<uint2 *>(p.out + orow * p.ld_o + (int64_t)hd * D + d) =
                                make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
                            if (p.lse && d == 0)
                                p.lse[orow * p.q_heads + hd] = sum_l == 0.0f ? -INFINITY : (m + log2_approx(sum_l)) * kLn2;
                        }
                    }
                }
            }
            g0 += steps;
            at += steps;
            if (at >= end) break;
            next_unit<NQ>(p, u);
        }
    }

    // ------------------------------- teardown -------------------------------
    __syncwarp();
    if (*abort_flag) __nanosleep(20000);   // let copies and products already issued drain before the memory is released
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    if (warp == kProductWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kTmemCols) : "memory");
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

template <int D, int NQ>
static cudaError_t configure_chunk()
{
    return cudaFuncSetAttribute(attn_chunk_kernel<D, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkShape<D, NQ>::kDynamic);
}
cudaError_t configure_attn_kernels()
{
    cudaError_t e = configure_chunk<128, 1>();
    if (e == cudaSuccess) e = configure_chunk<128, 2>();
    if (e == cudaSuccess) e = configure_chunk<64, 1>();
    if (e == cudaSuccess) e = configure_chunk<64, 2>();
    return e;
}

template <int D, int NQ>
static fp8_status_t launch_chunk(const fp8_ctx *ctx, AttnParams p, const fp8_kv_cache_t *c, cudaStream_t st)
{
    using L = ChunkShape<D, NQ>;
    const KvParams &kv = p.kv;
    const int64_t row_tiles = ((int64_t)kv.max_q_len * p.group + NQ * kTile - 1) / (NQ * kTile);
    const int64_t units = row_tiles * kv.seqs * kv.kv_heads, longest = ((int64_t)kv.max_kv_len + kTile - 1) / kTile;
    if (row_tiles * kv.seqs > INT32_MAX) return FP8_ERR_SHAPE;
    p.row_tiles = (int)row_tiles;
    // a CTA's share is at least four steps (see attn_chunk_kernel: shares below that spend more on joining than they save)
    p.min_share = 4;
    int64_t grid = (int64_t)ctx->sm_count * L::kResident;
    const int64_t most = (units * longest + p.min_share - 1) / p.min_share;
    if (most < grid) grid = most;
    if (grid * NQ > kAttnCounters || grid * 2 * NQ * L::kPart * 4 > (int64_t)ctx->partial_bytes) return FP8_ERR_UNSUPPORTED;
    CUtensorMap map;
    if (!encode_keys(ctx, &map, c)) return FP8_ERR_CUDA;
    count_launch();
    attn_chunk_kernel<D, NQ><<<(unsigned)grid, L::kThreads, L::kDynamic, st>>>(map, p);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

fp8_status_t attn_chunk(const fp8_ctx *ctx, const AttnParams &p, const fp8_kv_cache_t *c, int64_t rows, cudaStream_t st)
{
    if (c->head_dim == 128) return rows <= kTile ? launch_chunk<128, 1>(ctx, p, c, st) : launch_chunk<128, 2>(ctx, p, c, st);
    return rows <= kTile ? launch_chunk<64, 1>(ctx, p, c, st) : launch_chunk<64, 2>(ctx, p, c, st);
}

}  // namespace fp8lin
