// Attention over the paged FP8 cache for many query rows: chunks of a prompt, drafted tokens.
//
// A CTA takes 128 query rows of one key/value head (rows: token by token, the head's query heads side by side) and walks
// the cached tokens in tiles of 128, two products per tile on the 5th-generation tensor cores:
//   S = Q K^T   e4m3 x e4m3: the cache's key bytes are the operand as they lie (TMA, no conversion).  A query row is the
//               sum of two e4m3 numbers under one power of two, q 2^e = hi + lo (hi rounded to nearest, lo the rest):
//               eight significant bits together, so bf16 queries are exact unless 2^17 below their row's largest.  Two
//               e4m3 products cost what one bf16 product costs.
//   O += P V    bf16: a value 2^-d V8 is a bf16 number; four warps make them on their way into shared memory (once for the
//               128 rows).  P in its two bf16 terms is read from tensor memory, where it takes the place of the scores
//               that it came from, 32 tokens' terms side by side.
// Per CTA 256 of the 512 tensor-memory columns and half the shared memory: two CTAs share an SM, and while one waits for
// its softmax the other's products run.  Within a CTA the order is strict (S, softmax, O, next S), which also makes
// the rescaling of O safe without a barrier of its own: S of a tile is complete only after O of the tile before.
//
// Warps: 0-3 softmax (one row per thread) and output, 4-7 values and scaling biases, 8 keys (TMA), 9 products.
#include "attn_common.cuh"
#include "ptx.cuh"

namespace fp8lin {

constexpr int kTile = 128;                 // query rows, and tokens per step
constexpr int kChunkThreads = 320;
constexpr int kKStages = 2;

template <int D>
struct ChunkSmem {
    static constexpr int kQBytes = kTile * 2 * D;
    static constexpr int kKBytes = kTile * D;
    static constexpr int kVBytes = kTile * D * 2;
    static constexpr int kQ = 0;
    static constexpr int kK = kQ + kQBytes;
    static constexpr int kV = kK + kKStages * kKBytes;
    static constexpr int kScale = kV + kVBytes;              // [2][128] floats: 2^-b of a tile's keys
    static constexpr int kBar = kScale + 2 * kTile * 4;
    static constexpr int kNumBars = 2 * kKStages + 7;
    static constexpr int kTotal = kBar + kNumBars * 8 + 16;
    static constexpr int kDynamic = kTotal + 1024;           // slack to align the base to 1024 bytes
};
constexpr uint32_t kChunkTmemCols = 256;
constexpr uint32_t kTmemO = 128;           // columns 0..127: S, then P; 128..: O

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

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 2) attn_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const AttnParams p)
{
    using L = ChunkSmem<D>;
    extern __shared__ uint8_t smem_raw[];
    const KvParams &kv = p.kv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // ---- which rows, which tokens ----
    // the last rows of a sequence see most tokens under a causal mask: their tiles come first
    int id = blockIdx.x;
    const int split = id % p.splits;
    id /= p.splits;
    const int unit = id;
    const int h = id % kv.kv_heads;
    id /= kv.kv_heads;
    const int b = id % kv.seqs, row0 = (p.row_tiles - 1 - id / kv.seqs) * kTile;
    bool cut;
    const SeqShape s = seq_shape(kv, b, cut);
    if (cut && threadIdx.x == 0) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    const int rows = s.n * p.group - row0;            // rows of this tile (and beyond)
    if (rows <= 0) return;
    int see = s.len;                                  // tokens that the tile's last row sees
    if (p.causal) see = min(s.len, max(0, s.len - s.n + (row0 + min(rows, kTile) - 1) / p.group + 1));
    const int tiles = (see + kTile - 1) / kTile;
    const int parts = max(1, min(p.splits, tiles));
    if (split >= parts) return;
    const int tile0 = (int)((int64_t)tiles * split / parts), tile1 = (int)((int64_t)tiles * (split + 1) / parts);
    const int steps = tile1 - tile0;

    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem), bars = base + L::kBar;
    auto k_full = [&](int i) { return bars + 8u * i; };
    auto k_empty = [&](int i) { return bars + 8u * (kKStages + i); };
    const uint32_t s_full = bars + 8u * (2 * kKStages), p_full = s_full + 8u, v_full = s_full + 16u, v_empty = s_full + 24u,
                   o_full = s_full + 32u;
    auto sc_full = [&](int i) { return s_full + 40u + 8u * i; };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + L::kBar + L::kNumBars * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    volatile int *is_last = reinterpret_cast<volatile int *>(tmem_slot + 2);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kKStages; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); }
        mbar_init(s_full, 1);
        mbar_init(p_full, 4);
        mbar_init(v_full, 128);
        mbar_init(v_empty, 1);
        mbar_init(o_full, 1);
        for (int i = 0; i < 2; ++i) mbar_init(sc_full(i), 128);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kChunkTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    // ---- queries as two e4m3 terms, one row per thread of warps 0-3 ----
    float rc = 0.0f;        // |c| / the row's power of two
    int limit = 0;          // tokens that the row sees
    if (warp < 4) {
        const int r = threadIdx.x;
        const int tok = min((row0 + r) / p.group, s.n - 1), hq = h * p.group + (row0 + r) % p.group;
        const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (int64_t)(s.first + tok) * p.ld_q + (int64_t)hq * D);
        uint32_t m = 0;
        if (r < rows) {
#pragma unroll
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
        limit = s.len;
        if (p.causal) limit = min(s.len, max(0, s.len - s.n + (row0 + r) / p.group + 1));
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (r < rows) { x = src[2 * i]; y = src[2 * i + 1]; }
            const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = __uint_as_float(w[2 * j] << 16) * f, bb = __uint_as_float(w[2 * j] & 0xFFFF0000u) * f;
                const float cc = __uint_as_float(w[2 * j + 1] << 16) * f, d = __uint_as_float(w[2 * j + 1] & 0xFFFF0000u) * f;
                hi[j] = cvt_pair<FP8_E4>(bb, a) | (cvt_pair<FP8_E4>(d, cc) << 16);
                uint32_t h2[2];
                e4_to_f16(hi[j], h2[0], h2[1]);
                float back[4];
                unpack4<FP8_F16>(h2, back);
                lo[j] = cvt_pair<FP8_E4>(bb - back[1], a - back[0]) | (cvt_pair<FP8_E4>(d - back[3], cc - back[2]) << 16);
            }
            // D = 128: a row of hi, and 16 KB on its row of lo; D = 64: hi and lo side by side in one 128-byte row
            const int c_hi = i, c_lo = D == 128 ? i : i + 4;
            const uint32_t row = base + L::kQ + r * 128;
            sts16(row + ((c_hi ^ (r & 7)) << 4), hi[0], hi[1], hi[2], hi[3]);
            sts16(row + (D == 128 ? kTile * 128 : 0) + ((c_lo ^ (r & 7)) << 4), lo[0], lo[1], lo[2], lo[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int32_t *table = kv.table + (int64_t)b * kv.table_stride;
    const int last_page = (s.len - 1) >> kv.page_shift;      // of the sequence (only used where steps > 0)

    if (warp == 8) {
        // ------------------------------- keys -------------------------------
        const int per_tile = kTile >> kv.page_shift;          // pages of a tile: 1 to 8, one lane each
        auto page_of = [&](int tile) {
            const int j = tile * per_tile + lane;
            return lane < per_tile && j <= last_page ? __ldg(table + j) : -2;   // -2: nothing to load
        };
        int page = steps > 0 ? page_of(tile0) : -2;
        bool alive = true;
        for (int i = 0; i < steps && alive; ++i) {
            const int next = i + 1 < steps ? page_of(tile0 + i + 1) : -2;
            const int st = i % kKStages;
            const int j = (tile0 + i) * per_tile + lane;
            const bool load = lane < per_tile && j <= last_page;
            const int n = __popc(__ballot_sync(0xFFFFFFFFu, load));
            alive = mbar_wait(k_empty(st), ((i / kKStages) & 1u) ^ 1u, abort_flag, kv.d_status);
            alive = __all_sync(0xFFFFFFFFu, alive);
            if (!alive) break;
            if (lane == 0) mbar_expect_tx(k_full(st), (uint32_t)(n * D) << kv.page_shift);
            __syncwarp();
            // a page out of range is read as page 0; its tokens are marked non-finite by the warps of the values
            if (load)
                tma_load_page(base + L::kK + st * L::kKBytes + ((lane * D) << kv.page_shift), &map_k, k_full(st), h << kv.page_shift,
                              (unsigned)page < (unsigned)kv.pages ? page : 0);
            page = next;
        }
    } else if (warp == 9) {
        // ------------------------------- products -------------------------------
        if (lane == 0) {
            const uint32_t idesc_s = (1u << 4) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);          // e4m3 x e4m3
            const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) |
                                     ((uint32_t)(kTile >> 4) << 24);                                                       // bf16, B along N
            const uint64_t dv = desc_sw128(base + L::kV, kTile * 128);
            auto scores = [&](int i) {
                const int st = i % kKStages;
                const uint32_t k_addr = base + L::kK + st * L::kKBytes;
                const uint64_t dk = D == 128 ? desc_sw128(k_addr, 16) : desc_sw64(k_addr);
#pragma unroll
                for (int term = 0; term < 2; ++term) {
                    const uint64_t dq = D == 128 ? desc_sw128(base + L::kQ + term * kTile * 128, 16) : desc_sw128(base + L::kQ, 16) + 4u * term;
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) chunk_mma_f8(tmem, dq + 2u * k, dk + 2u * k, idesc_s, (term | k) ? 1u : 0u);
                }
                chunk_commit(k_empty(st));
                chunk_commit(s_full);
            };
            bool alive = steps > 0 && mbar_wait(k_full(0), 0, abort_flag, kv.d_status);
            if (alive) {
                chunk_fence_after();
                scores(0);
            }
            for (int i = 0; i < steps && alive; ++i) {
                alive = mbar_wait(v_full, i & 1u, abort_flag, kv.d_status) && mbar_wait(p_full, i & 1u, abort_flag, kv.d_status);
                if (!alive) break;
                chunk_fence_after();
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k) {      // 16 tokens: columns 8 (k % 2) of the 32 that hold 32 tokens
                    const uint32_t p1 = tmem + 32u * (k >> 1) + 8u * (k & 1);
                    chunk_mma_bf16_tmem(tmem + kTmemO, p1, dv + 128u * k, idesc_o, (i | k) ? 1u : 0u);
                    chunk_mma_bf16_tmem(tmem + kTmemO, p1 + 16u, dv + 128u * k, idesc_o, 1u);
                }
                chunk_commit(v_empty);
                if (i + 1 == steps) {
                    chunk_commit(o_full);
                } else {
                    alive = mbar_wait(k_full((i + 1) % kKStages), ((i + 1) / kKStages) & 1u, abort_flag, kv.d_status);
                    if (!alive) break;
                    chunk_fence_after();
                    scores(i + 1);
                }
            }
        }
    } else if (warp >= 4) {
        // ------------------------------- values and biases -------------------------------
        // A warp takes 32 tokens of each tile: lane (tok, c) = (lane / 4, lane % 4) of eight tokens at a time, 16 bytes.
        // Two neighbouring tokens and four pieces of 16 dimensions meet all banks once in each store of eight lanes.
        const int cw = warp - 4, sub = lane >> 2, c = lane & 3;
        constexpr int kHalves = D / 64, kLoads = 4 * kHalves;
        uint4 cur[kLoads], nxt[kLoads];
        int bk = 0, bv = 0, bk_n = 0, bv_n = 0;
        unsigned bad_pages = 0;
        auto request = [&](int tile, uint4 (&v)[kLoads], int &b_k, int &b_v) {
            // pages of the warp's tokens 0..15 and 16..31 (the same one unless pages hold 16 tokens)
            const int t0 = tile * kTile + cw * 32;
            int pg[2];
            bool ok[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int j = (t0 + 16 * i) >> kv.page_shift;
                ok[i] = t0 + 16 * i < s.len;
                pg[i] = ok[i] ? __ldg(table + j) : 0;
                if ((unsigned)pg[i] >= (unsigned)kv.pages) { pg[i] = -1; bad_pages = 1; }
            }
            const int in_page = (1 << kv.page_shift) - 1;
            const int64_t row_h = (int64_t)h << kv.page_shift;
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
                    const int64_t at = mine * kv.bias_stride + row_h + (tk & in_page);
                    b_k = kv.bk[at];
                    b_v = kv.bv[at];
                }
            }
        };
        if (steps > 0) request(tile0, cur, bk, bv);
        for (int i = 0; i < steps; ++i) {
            const int tile = tile0 + i;
            // the tile's factors: 2^-b of the keys for the softmax, 2^(120 - d) for the values
            const bool marked = bk == FP8_KV_BIAS_NONFINITE || bv == FP8_KV_BIAS_NONFINITE;
            const unsigned drop = __ballot_sync(0xFFFFFFFFu, marked);
            reinterpret_cast<float *>(smem + L::kScale)[(i & 1) * kTile + cw * 32 + lane] =
                marked ? __int_as_float(0x7FFFFFFF) : pow2_normal(min(126, -(bk + kv.delta)));
            const uint32_t factor = value_factor(bv + kv.delta), rest = value_factor_rest(bv + kv.delta);
            const bool two_steps = __any_sync(0xFFFFFFFFu, bv + kv.delta < -7);     // values beyond 2^15
            mbar_arrive(sc_full(i & 1));
            if (i + 1 < steps) request(tile + 1, nxt, bk_n, bv_n);
            if (i > 0) {
                const bool ok = mbar_wait(v_empty, (i - 1) & 1u, abort_flag, kv.d_status);
                if (!__all_sync(0xFFFFFFFFu, ok)) break;
            }
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
                const uint32_t row = base + L::kV + half * (kTile * 128) + tk * 128;
                sts16(row + (((2 * c) ^ (tk & 7)) << 4), w[0], w[1], w[2], w[3]);
                sts16(row + (((2 * c + 1) ^ (tk & 7)) << 4), w[4], w[5], w[6], w[7]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(v_full);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) cur[k] = nxt[k];
            bk = bk_n;
            bv = bv_n;
        }
        if (bad_pages) raise_flags(kv.d_status, FP8_FLAG_BAD_INDEX);
    } else {
        // ------------------------------- softmax -------------------------------
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        const bool active = warp * 32 < rows;
        const int least = __shfl_sync(0xFFFFFFFFu, limit, 0);      // what the warp's first row sees: the least of its rows
        float top = kNoMax;
        f32x2 sum = pack2(0.0f, 0.0f);
        const f32x2 rc2 = pack2(rc, rc);
        for (int i = 0; i < steps; ++i) {
            const int t0 = (tile0 + i) * kTile;
            bool ok = mbar_wait(s_full, i & 1u, abort_flag, kv.d_status);
            ok = ok && mbar_wait(sc_full(i & 1), (i >> 1) & 1u, abort_flag, kv.d_status);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            chunk_fence_after();
            if (active) {
                const uint32_t sc = base + L::kScale + (i & 1) * (kTile * 4);
                const bool mask = t0 + kTile > least;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    uint32_t x[32];
                    tmem_load32(lanes + 32u * ch, x);
                    tmem_wait_ld();
                    // u = 2^-b (q . K8), s = rc u
                    f32x2 u[16];
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        f32x2 f0, f1;
                        lds_pairs(sc + (ch * 32 + 2 * k) * 4, f0, f1);
                        u[k] = mul2(pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), f0);
                        u[k + 1] = mul2(pack2(__uint_as_float(x[2 * k + 2]), __uint_as_float(x[2 * k + 3])), f1);
                    }
                    if (mask) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float lo, hi;
                            unpack2(u[k], lo, hi);
                            const int j = t0 + ch * 32 + 2 * k;
                            if (j >= limit) lo = -INFINITY;
                            if (j + 1 >= limit) hi = -INFINITY;
                            u[k] = pack2(lo, hi);
                        }
                    }
                    float m = -INFINITY;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float lo, hi;
                        unpack2(u[k], lo, hi);
                        m = fmaxf(m, fmaxf(lo, hi));
                    }
                    m *= rc;
                    if (__any_sync(0xFFFFFFFFu, m > top + kSlack)) {
                        // rare: move M (by a whole number of powers of two, exact for bf16 too), and bring to it what has
                        // been summed and the weights of this tile already written
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
                    }
                    const f32x2 minus = pack2(-top, -top);
                    uint32_t ph[32];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float lo, hi;
                        unpack2(fma2(u[k], rc2, minus), lo, hi);
                        lo = exp2_approx(lo);
                        hi = exp2_approx(hi);
                        sum = add2(sum, pack2(lo, hi));
                        split_bf16(lo, hi, ph[k], ph[16 + k]);
                    }
                    tmem_store32(lanes + 32u * ch, ph);
                }
                tmem_wait_st();
            }
            chunk_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);
        }
        // ------------------------------- output -------------------------------
        float total;
        {
            float lo, hi;
            unpack2(sum, lo, hi);
            total = lo + hi;
        }
        if (steps > 0) {
            mbar_wait(o_full, 0, abort_flag, kv.d_status);
            __syncwarp();
            chunk_fence_after();
        }
        const int r = threadIdx.x;
        const bool mine = r < rows;
        const int64_t out_row = s.first + min((row0 + r) / p.group, s.n - 1);
        const int head = h * p.group + (row0 + r) % p.group;
        uint16_t *dst = p.out + out_row * p.ld_o + (int64_t)head * D;
        float *lse = p.lse ? p.lse + out_row * p.q_heads + head : nullptr;
        if (parts == 1) {
            const float inv = total == 0.0f ? 0.0f : 1.0f / total;
            if (active) {
#pragma unroll
                for (int ch = 0; ch < D / 32; ++ch) {
                    uint32_t x[32];
                    if (steps > 0) {
                        tmem_load32(lanes + kTmemO + 32u * ch, x);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = 0u;
                    }
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
                if (mine && lse) *lse = total == 0.0f ? -INFINITY : (top + log2_approx(total)) * kLn2;
            }
        } else {
            // a part of the row's tokens: unscaled sums and statistics to the workspace, joined in order by the last
            constexpr int64_t kPart = kTile * (D + 2);
            float *slot = p.part + ((int64_t)unit * p.splits + split) * kPart;
            if (active) {
#pragma unroll
                for (int ch = 0; ch < D / 32; ++ch) {
                    uint32_t x[32];
                    tmem_load32(lanes + kTmemO + 32u * ch, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (mine) *reinterpret_cast<uint4 *>(slot + r * D + ch * 32 + 4 * k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    __syncwarp();
                }
                if (mine) { slot[kTile * D + r] = top; slot[kTile * D + kTile + r] = total; }
            }
            __threadfence();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (threadIdx.x == 0) *is_last = atomicAdd(p.count + unit, 1u) == (unsigned)(parts - 1);
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (*is_last) {
                __threadfence();
                if (threadIdx.x == 0) p.count[unit] = 0u;
                const float *all = p.part + (int64_t)unit * p.splits * kPart;
                // lanes side by side along a row: 32 lanes take 128 dimensions of one row at a time
                const int per_row = D / 4, row_step = 128 / per_row;
                for (int rr = threadIdx.x / per_row; rr < min(rows, kTile); rr += row_step) {
                    const int d = threadIdx.x % per_row * 4;
                    float m = kNoMax;
                    for (int k = 0; k < parts; ++k) m = fmaxf(m, __ldcg(all + k * kPart + kTile * D + rr));
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    float l = 0.0f;
                    for (int k = 0; k < parts; ++k) {
                        const float *src = all + k * kPart;
                        const float f = exp2_approx(__ldcg(src + kTile * D + rr) - m);
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(src + rr * D + d));
                        v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
                        l = fmaf(__ldcg(src + kTile * D + kTile + rr), f, l);
                    }
                    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                    const int64_t orow = s.first + (row0 + rr) / p.group;
                    const int hd = h * p.group + (row0 + rr) % p.group;
                    *reinterpret_cast<uint2 *>(p.out + orow * p.ld_o + (int64_t)hd * D + d) =
                        make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
                    if (p.lse && d == 0)
                        p.lse[orow * p.q_heads + hd] = l == 0.0f ? -INFINITY : (m + log2_approx(l)) * kLn2;
                }
            }
        }
    }

    // ------------------------------- teardown -------------------------------
    __syncwarp();
    if (*abort_flag) __nanosleep(20000);   // let copies and products already issued drain before the memory is released
    chunk_fence_before();
    __syncthreads();
    chunk_fence_after();
    if (warp == 9)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kChunkTmemCols) : "memory");
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
    cudaError_t e = cudaFuncSetAttribute(attn_chunk_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkSmem<128>::kDynamic);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(attn_chunk_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkSmem<64>::kDynamic);
}

fp8_status_t attn_chunk(const fp8_ctx *ctx, AttnParams p, const fp8_kv_cache_t *c, cudaStream_t st)
{
    const KvParams &kv = p.kv;
    const int64_t row_tiles = ((int64_t)kv.max_q_len * p.group + kTile - 1) / kTile;
    const int64_t units = row_tiles * kv.seqs * kv.kv_heads;
    // Contexts are cut into parts where the tiles alone leave places empty: as many parts as fill one round of two CTAs
    // per SM, at least two steps each.
    const int64_t places = 2 * (int64_t)ctx->sm_count, longest = ((int64_t)kv.max_kv_len + kTile - 1) / kTile;
    int64_t splits = places / units;
    if (splits > longest / 2) splits = longest / 2;
    if (splits < 1) splits = 1;
    if (row_tiles > INT32_MAX || units * splits > INT32_MAX) return FP8_ERR_SHAPE;
    if (splits > 1 && (units > kAttnCounters || units * splits * kTile * (c->head_dim + 2) * 4 > (int64_t)ctx->partial_bytes)) splits = 1;
    p.row_tiles = (int)row_tiles;
    p.splits = (int)splits;
    CUtensorMap map;
    if (!encode_keys(ctx, &map, c)) return FP8_ERR_CUDA;
    count_launch();
    if (c->head_dim == 128) attn_chunk_kernel<128><<<(unsigned)(units * splits), kChunkThreads, ChunkSmem<128>::kDynamic, st>>>(map, p);
    else attn_chunk_kernel<64><<<(unsigned)(units * splits), kChunkThreads, ChunkSmem<64>::kDynamic, st>>>(map, p);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

}  // namespace fp8lin
