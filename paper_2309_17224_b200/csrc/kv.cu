// Quantising keys and values into the paged FP8 cache, and reading them back.
//
// A row (one token, one key/value head) is head_dim numbers: 8 to 32 lanes hold it, 16 bytes each, its amax is a few
// shuffles, and the bytes leave from the same registers: one pass over memory, head_dim * (size + 1) + 1 bytes a row.
// A warp takes one token and a few of its heads, keys and values together (the walk row -> sequence -> page is done once,
// and its three dependent loads overlap the loads of the numbers), and ends: blocks that come and go fill the SMs evenly,
// where a resident grid that walks the tokens loses the last, partly filled round (8192 tokens of 32 heads of 128: 41.8
// against 43.9 us; 65536 tokens of 8 heads read: 53.9 against 57.3, both when this was chosen).  Measured from a graph: the
// first 41.7 us for 202 MB (FP16 41.5, FP32 65.3 for 336 MB), bound by instruction issue; the second 52.8 us for 320 MB (FP32
// 86.1 for 533 MB), bound by memory.
// Four heads one after the other per lane group, 128 bytes in flight per lane; two where that would leave the SMs half
// empty (16 tokens of 8 heads: 3.1 against 4.2 us; 8192 tokens of 32 heads: 44.2 against 41.8).
#include "kv_common.cuh"

namespace fp8lin {

template <int DT, int D, int UNROLL>
struct RowShape {
    static constexpr int kElems = 16 / InType<DT>::kBytes;       // numbers per lane
    static constexpr int kLanes = D / kElems;                    // lanes per row
    static constexpr int kRowsPerWarp = 32 / kLanes;             // heads side by side in a warp
    static constexpr int kUnroll = UNROLL;                       // ... and one after the other
    static constexpr int kHeads = kRowsPerWarp * kUnroll;        // heads of a warp's task
};

// Largest magnitude (as FP32 bits: NaN above infinity above every number) of one lane's 16 bytes.  Magnitudes of one type
// are in the order of their bits, so 16-bit types are compared two at a time and only the largest is converted.
template <int DT>
__device__ __forceinline__ uint32_t lane_amax_bits(const uint32_t (&w)[4])
{
    if (DT == FP8_F32) return max(max(w[0] & 0x7FFFFFFFu, w[1] & 0x7FFFFFFFu), max(w[2] & 0x7FFFFFFFu, w[3] & 0x7FFFFFFFu));
    const uint32_t m2 = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    const uint32_t m = max(m2 & 0xFFFFu, m2 >> 16);
    if (DT == FP8_BF16) return m << 16;
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)m));
    return __float_as_uint(f);
}

// Quantise the row that kLanes neighbouring lanes hold; every lane gets its bytes (kElems of them) and the row's bias.
template <int DT, int D>
__device__ __forceinline__ int quantise_row(const uint4 v, int conv, int delta, uint32_t (&out)[2], unsigned &flags)
{
    using R = RowShape<DT, D, 1>;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = lane_amax_bits<DT>(w);
#pragma unroll
    for (int s = R::kLanes / 2; s > 0; s >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));
    const int bias = max(-127, min(FP8_KV_BIAS_MAX, bias_from_amax_bits(m, FP8_E4, conv, 0, &flags)));
    const float scale = pow2_normal(bias + delta);   // -121 .. 65: one normal factor
    // the largest magnitude clips first; a NaN hides it
    if (clips<FP8_E4>(__uint_as_float(m) * scale)) flags |= FP8_FLAG_SATURATED;
    const bool hidden = m > 0x7F800000u;
#pragma unroll
    for (int i = 0; i < R::kElems / 4; ++i) {
        float f[4];
        unpack4<DT>(w + i * InType<DT>::kWords4, f);
        if (hidden && (clips<FP8_E4>(f[0] * scale) || clips<FP8_E4>(f[1] * scale) || clips<FP8_E4>(f[2] * scale) || clips<FP8_E4>(f[3] * scale)))
            flags |= FP8_FLAG_SATURATED;
        out[i] = cvt_pair<FP8_E4>(f[1] * scale, f[0] * scale) | (cvt_pair<FP8_E4>(f[3] * scale, f[2] * scale) << 16);
    }
    return m >= 0x7F800000u ? FP8_KV_BIAS_NONFINITE : bias;
}

template <int DT, int D, int UNROLL>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvParams p, const uint8_t *__restrict__ k, const uint8_t *__restrict__ v,
                                                        int64_t row_k, int64_t row_v)
{
    using R = RowShape<DT, D, UNROLL>;
    const int lane = threadIdx.x & 31, part = lane % R::kLanes, sub = lane / R::kLanes;
    const int h0 = blockIdx.y * R::kHeads + sub;
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= p.tokens) return;
    uint4 xk[R::kUnroll], xv[R::kUnroll];
#pragma unroll
    for (int u = 0; u < R::kUnroll; ++u) {
        const int h = h0 + u * R::kRowsPerWarp;
        xk[u] = xv[u] = make_uint4(0u, 0u, 0u, 0u);
        if (h < p.kv_heads) {
            const int64_t at = (int64_t)h * (D * InType<DT>::kBytes) + part * 16;
            xk[u] = load_stream(k + t * row_k + at);
            xv[u] = load_stream(v + t * row_v + at);
        }
    }
    // looked up while the numbers are on their way
    int page = 0, off = 0;
    const RowPlace place = place_of_row(p, (int)t, lane, page, off);
    if (place != kWritten) {
        if (place == kBad && lane == 0) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
        return;
    }
    unsigned flags = 0;
#pragma unroll
    for (int u = 0; u < R::kUnroll; ++u) {
        const int h = h0 + u * R::kRowsPerWarp;
        uint32_t ck[2], cv[2];
        unsigned met = 0;
        const int bk = quantise_row<DT, D>(xk[u], p.conv, p.delta, ck, met);
        const int bv = quantise_row<DT, D>(xv[u], p.conv, p.delta, cv, met);
        if (h >= p.kv_heads) continue;
        flags |= met;
        const int64_t row = ((int64_t)h << p.page_shift) + off;
        const int64_t at = page * p.page_stride + row * D + part * R::kElems;
        if (R::kElems == 8) {
            *reinterpret_cast<uint2 *>(p.k8 + at) = make_uint2(ck[0], ck[1]);
            *reinterpret_cast<uint2 *>(p.v8 + at) = make_uint2(cv[0], cv[1]);
        } else {
            *reinterpret_cast<uint32_t *>(p.k8 + at) = ck[0];
            *reinterpret_cast<uint32_t *>(p.v8 + at) = cv[0];
        }
        if (part == 0) {
            p.bk[page * p.bias_stride + row] = (int8_t)bk;
            p.bv[page * p.bias_stride + row] = (int8_t)bv;
        }
    }
    flags = __reduce_or_sync(0xFFFFFFFFu, flags);
    if (lane == 0 && flags) raise_flags(p.d_status, flags);
}

// Four E4 bytes as numbers (exact).
__device__ __forceinline__ void unpack_e4(uint32_t w, float (&f)[4])
{
    uint32_t lo, hi;
    asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }" : "=r"(lo), "=r"(hi) : "r"(w));
    const uint32_t h[2] = {lo, hi};
    unpack4<FP8_F16>(h, f);
}

// One lane's kElems bytes as kElems numbers of type DT, times the power of two, rounded once.
template <int DT>
__device__ __forceinline__ uint4 dequantise(const uint32_t (&c)[2], float scale)
{
    float f[8];
    unpack_e4(c[0], *reinterpret_cast<float(*)[4]>(f));
    if (DT != FP8_F32) unpack_e4(c[1], *reinterpret_cast<float(*)[4]>(f + 4));
#pragma unroll
    for (int i = 0; i < (DT == FP8_F32 ? 4 : 8); ++i) f[i] *= scale;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DT == FP8_F32) w[i] = __float_as_uint(f[i]);
        else if (DT == FP8_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT, int D, int UNROLL>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvParams p, uint8_t *__restrict__ k, uint8_t *__restrict__ v, int64_t row_k,
                                                      int64_t row_v)
{
    using R = RowShape<DT, D, UNROLL>;
    const int lane = threadIdx.x & 31, part = lane % R::kLanes, sub = lane / R::kLanes;
    const int h0 = blockIdx.y * R::kHeads + sub;
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= p.tokens) return;
    int page = 0, off = 0;
    const RowPlace place = place_of_row(p, (int)t, lane, page, off);
    if (place == kBad && lane == 0) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
    uint32_t c[2][R::kUnroll][2] = {};
    int b[2][R::kUnroll] = {};
#pragma unroll
    for (int u = 0; u < R::kUnroll; ++u) {
        const int h = h0 + u * R::kRowsPerWarp;
        if (place != kWritten || h >= p.kv_heads) continue;
        const int64_t row = ((int64_t)h << p.page_shift) + off;
        const int64_t at = page * p.page_stride + row * D + part * R::kElems;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint8_t *src = (s ? p.v8 : p.k8) + at;
            if (!(s ? v : k)) continue;
            if (R::kElems == 8) {
                const uint2 x = *reinterpret_cast<const uint2 *>(src);
                c[s][u][0] = x.x;
                c[s][u][1] = x.y;
            } else {
                c[s][u][0] = *reinterpret_cast<const uint32_t *>(src);
            }
            b[s][u] = (s ? p.bv : p.bk)[page * p.bias_stride + row];
        }
    }
#pragma unroll
    for (int u = 0; u < R::kUnroll; ++u) {
        const int h = h0 + u * R::kRowsPerWarp;
        if (h >= p.kv_heads) continue;
        const int64_t at = (int64_t)h * (D * InType<DT>::kBytes) + part * 16;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint8_t *dst = s ? v : k;
            if (!dst) continue;
            // -65 .. 126: one normal factor (no finite row has a bias below -121)
            const float scale = pow2_normal(min(126, -(applied_bias(b[s][u]) + p.delta)));
            __stcs(reinterpret_cast<uint4 *>(dst + t * (s ? row_v : row_k) + at), dequantise<DT>(c[s][u], scale));
        }
    }
}

// Blocks of eight warps, a warp per token and group of heads.
template <int DT, int D, int UNROLL>
static dim3 kv_grid(const KvParams &p)
{
    return dim3((unsigned)(((int64_t)p.tokens + 7) / 8), (unsigned)((p.kv_heads + RowShape<DT, D, UNROLL>::kHeads - 1) / RowShape<DT, D, UNROLL>::kHeads));
}
// Whether four heads per lane group still give every SM its 32 resident warps.
template <int DT, int D>
static bool kv_long(const fp8_ctx *ctx, const KvParams &p)
{
    const dim3 g = kv_grid<DT, D, 4>(p);
    return (int64_t)g.x * g.y * 8 >= (int64_t)ctx->sm_count * 32;
}

template <int DT, int D>
static fp8_status_t launch_append(const fp8_ctx *ctx, const KvParams &p, const void *k, const void *v, int64_t ld_k, int64_t ld_v,
                                  cudaStream_t st)
{
    const uint8_t *k8 = static_cast<const uint8_t *>(k), *v8 = static_cast<const uint8_t *>(v);
    const int64_t row_k = ld_k * InType<DT>::kBytes, row_v = ld_v * InType<DT>::kBytes;
    count_launch();
    if (kv_long<DT, D>(ctx, p)) kv_append_kernel<DT, D, 4><<<kv_grid<DT, D, 4>(p), 256, 0, st>>>(p, k8, v8, row_k, row_v);
    else kv_append_kernel<DT, D, 2><<<kv_grid<DT, D, 2>(p), 256, 0, st>>>(p, k8, v8, row_k, row_v);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

template <int DT, int D>
static fp8_status_t launch_read(const fp8_ctx *ctx, const KvParams &p, void *k, void *v, int64_t ld_k, int64_t ld_v, cudaStream_t st)
{
    uint8_t *k8 = static_cast<uint8_t *>(k), *v8 = static_cast<uint8_t *>(v);
    const int64_t row_k = ld_k * InType<DT>::kBytes, row_v = ld_v * InType<DT>::kBytes;
    count_launch();
    if (kv_long<DT, D>(ctx, p)) kv_read_kernel<DT, D, 4><<<kv_grid<DT, D, 4>(p), 256, 0, st>>>(p, k8, v8, row_k, row_v);
    else kv_read_kernel<DT, D, 2><<<kv_grid<DT, D, 2>(p), 256, 0, st>>>(p, k8, v8, row_k, row_v);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

static fp8_status_t check_rows(const fp8_kv_cache_t *c, const void *x, int dt, int64_t ld)
{
    if (ld < (int64_t)c->kv_heads * c->head_dim) return FP8_ERR_SHAPE;
    if (c->kv_heads > 65535) return FP8_ERR_SHAPE;   // (groups of heads are the grid's second dimension)
    if (!kv_aligned16(x) || (ld * (dt == FP8_F32 ? 4 : 2)) % 16 != 0) return FP8_ERR_ALIGN;
    return FP8_OK;
}

}  // namespace fp8lin

#define FP8LIN_BY_TYPE(LAUNCH, ...)                                                                                                    \
    (c->head_dim == 128                                                                                                                \
         ? (dt == FP8_BF16 ? LAUNCH<FP8_BF16, 128>(__VA_ARGS__)                                                                        \
                           : dt == FP8_F16 ? LAUNCH<FP8_F16, 128>(__VA_ARGS__) : LAUNCH<FP8_F32, 128>(__VA_ARGS__))                    \
         : (dt == FP8_BF16 ? LAUNCH<FP8_BF16, 64>(__VA_ARGS__)                                                                         \
                           : dt == FP8_F16 ? LAUNCH<FP8_F16, 64>(__VA_ARGS__) : LAUNCH<FP8_F32, 64>(__VA_ARGS__)))

extern "C" {

fp8_status_t fp8_kv_append(fp8_ctx *ctx, const fp8_kv_cache_t *c, const fp8_seq_batch_t *batch, const void *k, const void *v,
                           fp8_dtype_t dt, int64_t ld_k, int64_t ld_v, fp8_conv_t conv, void *stream)
{
    using namespace fp8lin;
    fp8_status_t s = check_kv(ctx, c, batch, (int)conv);
    if (s != FP8_OK) return s;
    if (!k || !v) return FP8_ERR_NULL;
    if ((int)dt < 0 || (int)dt > 2) return FP8_ERR_DTYPE;
    if ((s = check_rows(c, k, (int)dt, ld_k)) != FP8_OK || (s = check_rows(c, v, (int)dt, ld_v)) != FP8_OK) return s;
    const KvParams p = make_kv_params(ctx, c, batch, (int)conv);
    return FP8LIN_BY_TYPE(launch_append, ctx, p, k, v, ld_k, ld_v, (cudaStream_t)stream);
}

fp8_status_t fp8_kv_read(fp8_ctx *ctx, const fp8_kv_cache_t *c, const fp8_seq_batch_t *batch, void *k, void *v, fp8_dtype_t dt,
                         int64_t ld_k, int64_t ld_v, fp8_conv_t conv, void *stream)
{
    using namespace fp8lin;
    fp8_status_t s = check_kv(ctx, c, batch, (int)conv);
    if (s != FP8_OK) return s;
    if (!k && !v) return FP8_ERR_NULL;
    if ((int)dt < 0 || (int)dt > 2) return FP8_ERR_DTYPE;
    if (k && (s = check_rows(c, k, (int)dt, ld_k)) != FP8_OK) return s;
    if (v && (s = check_rows(c, v, (int)dt, ld_v)) != FP8_OK) return s;
    const KvParams p = make_kv_params(ctx, c, batch, (int)conv);
    return FP8LIN_BY_TYPE(launch_read, ctx, p, k, v, ld_k, ld_v, (cudaStream_t)stream);
}

}  // extern "C"
