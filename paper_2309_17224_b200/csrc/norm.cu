// Layer norm and its root-mean-square form, forward (with the residual sum, and the E4 bytes and amax of the output) and
// backward.
#include "fp8_norm.h"
#include "kv_common.cuh"
#include "row_common.cuh"

namespace fp8lin {

constexpr int kNormThreads = 256;
constexpr int kMaxCols = 1 << 30;

struct NormFwd {
    const void *x, *res, *w, *b;
    void *h, *y;
    float *mean, *rstd;
    uint8_t *y8;
    const int32_t *bias;   // of y8: given, or what the first pass left
    int64_t rows, ld_x, ld_res, ld_h, ld_y;
    int cols, w_dt, delta, layer;
    float eps, inv_cols;
    AmaxSink sink;
};

template <int DT>
__device__ __forceinline__ float normalised(const NormFwd &p, float h, float mean, float rstd, int j)
{
    float v = __fmul_rn(__fsub_rn(h, mean), rstd);
    const float w = p.w ? load_any(p.w, p.w_dt, j) : 1.0f, b = p.b ? load_any(p.b, p.w_dt, j) : 0.0f;
    return element_value<DT>(element_bits<DT>(__fmaf_rn(v, w, b)));
}

// Any sizes and alignment: a block per row, three walks over it.  CAST_ONLY: the statistics are there, bytes are wanted.
template <int DT, bool CAST_ONLY>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_any_kernel(const NormFwd p)
{
    __shared__ float part[2][kNormThreads / 32];
    uint32_t key = 0;
    bool sat = false;
    const bool bytes = p.y8 && p.bias;
    Pow2Pair scale = {1.0f, 1.0f};
    if (bytes) scale = make_pow2_pair(*p.bias + p.delta);
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        auto sum_at = [&](int j) {
            float v = load1<DT>(p.x, r * p.ld_x + j);
            if (p.res) v = element_value<DT>(element_bits<DT>(v + load1<DT>(p.res, r * p.ld_res + j)));
            return v;
        };
        auto h_at = [&](int j) { return p.h ? load1<DT>(p.h, r * p.ld_h + j) : sum_at(j); };
        float mean = 0.0f, rstd;
        if (CAST_ONLY) {
            mean = p.layer ? p.mean[r] : 0.0f;
            rstd = p.rstd[r];
        } else {
            float s = 0.0f;
            for (int j = threadIdx.x; j < p.cols; j += kNormThreads) {
                const float v = sum_at(j);
                if (p.h) store_bits<DT>(p.h, r * p.ld_h + j, element_bits<DT>(v));
                s += v;
            }
            s = block_sum<kNormThreads>(s, part[0]);
            if (p.layer) mean = s * p.inv_cols;
            float q = 0.0f;
            for (int j = threadIdx.x; j < p.cols; j += kNormThreads) {
                const float d = h_at(j) - mean;
                q = __fmaf_rn(d, d, q);
            }
            q = block_sum<kNormThreads>(q, part[1]);
            rstd = 1.0f / sqrtf(__fmaf_rn(q, p.inv_cols, p.eps));
            if (threadIdx.x == 0) {
                if (p.mean) p.mean[r] = mean;
                if (p.rstd) p.rstd[r] = rstd;
            }
        }
        if (p.y || bytes || p.sink.slot) {
            for (int j = threadIdx.x; j < p.cols; j += kNormThreads) {
                const float v = normalised<DT>(p, h_at(j), mean, rstd, j);
                key = max(key, magnitude_key(v));
                if (p.y && !CAST_ONLY) store_bits<DT>(p.y, r * p.ld_y + j, element_bits<DT>(v));
                if (bytes) {
                    const float z = v * scale.first * scale.second;
                    sat = sat || clips<FP8_E4>(z);
                    p.y8[r * p.cols + j] = (uint8_t)(cvt_pair<FP8_E4>(0.0f, z) & 0xFFu);
                }
            }
        }
    }
    if (sat) raise_flags(p.sink.d_status, FP8_FLAG_SATURATED);
    if (!CAST_ONLY) sink_amax(key, p.sink);
}

struct NormBwd {
    const void *dy, *h, *dh, *w;
    const float *mean, *rstd;
    void *dx;
    float *part_w, *part_b;   // [blocks][cols], or NULL
    int64_t rows, ld_dy, ld_h, ld_dh, ld_dx;
    int cols, w_dt, layer;
    float inv_cols;
    AmaxSink sink;
};

// Any sizes and alignment: a block per row at a time; the rows of a block add up in its own line of the workspace.
template <int DT>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_any_kernel(const NormBwd p)
{
    __shared__ float part[2][2][kNormThreads / 32];
    uint32_t key = 0;
    int turn = 0;
    float *pw = p.part_w ? p.part_w + (int64_t)blockIdx.x * p.cols : nullptr;
    float *pb = p.part_b ? p.part_b + (int64_t)blockIdx.x * p.cols : nullptr;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn ^= 1) {
        const float mean = p.layer ? p.mean[r] : 0.0f, rstd = p.rstd[r];
        const bool first = r == blockIdx.x;
        float s1 = 0.0f, s2 = 0.0f;
        for (int j = threadIdx.x; j < p.cols; j += kNormThreads) {
            const float dy = load1<DT>(p.dy, r * p.ld_dy + j), xh = (load1<DT>(p.h, r * p.ld_h + j) - mean) * rstd;
            const float g = p.w ? dy * load_any(p.w, p.w_dt, j) : dy;
            s1 += g;
            s2 = __fmaf_rn(g, xh, s2);
            if (pw) pw[j] = __fmaf_rn(dy, xh, first ? 0.0f : pw[j]);
            if (pb) pb[j] = first ? dy : pb[j] + dy;
        }
        if (!p.dx) continue;
        const float c1 = p.layer ? block_sum<kNormThreads>(s1, part[turn][0]) * p.inv_cols : 0.0f;
        const float c2 = block_sum<kNormThreads>(s2, part[turn][1]) * p.inv_cols;
        for (int j = threadIdx.x; j < p.cols; j += kNormThreads) {
            const float dy = load1<DT>(p.dy, r * p.ld_dy + j), xh = (load1<DT>(p.h, r * p.ld_h + j) - mean) * rstd;
            const float g = p.w ? dy * load_any(p.w, p.w_dt, j) : dy;
            float v = rstd * (g - c1 - xh * c2);
            if (p.dh) v += load1<DT>(p.dh, r * p.ld_dh + j);
            const uint32_t bits = element_bits<DT>(v);
            key = max(key, magnitude_key(element_value<DT>(bits)));
            store_bits<DT>(p.dx, r * p.ld_dx + j, bits);
        }
    }
    sink_amax(key, p.sink);
}

// Sums of the blocks' lines, in their order: 32 columns a block, eight lines at a time.
__global__ void __launch_bounds__(256) norm_bwd_sum_kernel(const float *part_w, const float *part_b, int lines, int cols, int w_dt,
                                                           void *dw, void *db)
{
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, j = blockIdx.x * 32 + lane;
    const float *part = blockIdx.y ? part_b : part_w;
    void *out = blockIdx.y ? db : dw;
    if (!out) return;
    float s = 0.0f;
    if (j < cols)
        for (int i = group; i < lines; i += 8) s += part[(int64_t)i * cols + j];
    sums[group][lane] = s;
    __syncthreads();
    if (group != 0 || j >= cols) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sums[i][lane];
    if (w_dt == FP8_F32) store_bits<FP8_F32>(out, j, element_bits<FP8_F32>(s));
    else if (w_dt == FP8_BF16) store_bits<FP8_BF16>(out, j, element_bits<FP8_BF16>(s));
    else store_bits<FP8_F16>(out, j, element_bits<FP8_F16>(s));
}

static unsigned blocks_for_rows(const fp8_ctx *ctx, int64_t rows, int per_sm)
{
    const int64_t most = (int64_t)ctx->sm_count * per_sm;
    return (unsigned)(rows < most ? rows : most);
}

template <int DT>
static void launch_fwd(const fp8_ctx *ctx, NormFwd p, bool two, cudaStream_t st)
{
    const unsigned grid = blocks_for_rows(ctx, p.rows, 8);
    const int32_t *bias = p.bias;
    if (two) p.bias = nullptr;
    count_launch();
    norm_fwd_any_kernel<DT, false><<<grid, kNormThreads, 0, st>>>(p);
    if (two) {
        p.bias = bias;
        count_launch();
        norm_fwd_any_kernel<DT, true><<<grid, kNormThreads, 0, st>>>(p);
    }
}

template <int DT>
static void launch_bwd(const fp8_ctx *ctx, const NormBwd &p, unsigned grid, cudaStream_t st)
{
    count_launch();
    norm_bwd_any_kernel<DT><<<grid, kNormThreads, 0, st>>>(p);
}

}  // namespace fp8lin

extern "C" {

fp8_status_t fp8_norm_fwd(fp8_ctx *ctx, const fp8_norm_fwd_t *a, void *stream)
{
    using namespace fp8lin;
    if (!ctx || !a || !a->x) return FP8_ERR_NULL;
    if (!a->h && !a->y && !a->d_mean && !a->d_rstd && !a->y8 && !a->d_amax && !a->d_bias_out) return FP8_ERR_NULL;
    if (a->y8 && !a->d_bias_in && !a->d_bias_out) return FP8_ERR_NULL;
    if (a->kind < 0 || a->kind > 1 || a->dt < 0 || a->dt > 2 || a->w_dt < 0 || a->w_dt > 2 || a->conv < 0 || a->conv > 1)
        return FP8_ERR_DTYPE;
    if ((a->weight || a->bias_vec) && a->w_dt != a->dt && a->w_dt != FP8_F32) return FP8_ERR_UNSUPPORTED;
    if (a->rows <= 0 || a->cols <= 0 || a->cols > kMaxCols || !(a->eps >= 0.0f && a->eps <= FLT_MAX)) return FP8_ERR_SHAPE;
    if (a->ld_x < a->cols || (a->residual && a->ld_residual < a->cols) || (a->h && a->ld_h < a->cols) || (a->y && a->ld_y < a->cols))
        return FP8_ERR_SHAPE;
    if (!element_aligned(a->x, a->dt) || !element_aligned(a->residual, a->dt) || !element_aligned(a->h, a->dt) ||
        !element_aligned(a->y, a->dt) || !element_aligned(a->weight, a->w_dt) || !element_aligned(a->bias_vec, a->w_dt) ||
        !element_aligned(a->d_mean, FP8_F32) || !element_aligned(a->d_rstd, FP8_F32) || !element_aligned(a->d_bias_in, FP8_F32) ||
        !element_aligned(a->d_amax, FP8_F32) || !element_aligned(a->d_bias_out, FP8_F32))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const bool two = a->y8 && !a->d_bias_in;
    // the second pass starts from the statistics of the first
    if (two && (!a->d_rstd || (a->kind == FP8_NORM_LAYER && !a->d_mean))) return FP8_ERR_NULL;
    NormFwd p = {a->x, a->residual, a->weight, a->bias_vec, a->h, a->y, a->d_mean, a->d_rstd, a->y8, two ? a->d_bias_out : a->d_bias_in,
                 a->rows, a->ld_x, a->ld_residual, a->ld_h, a->ld_y, (int)a->cols, a->w_dt, format_delta(FP8_E4, a->conv),
                 a->kind == FP8_NORM_LAYER, a->eps, 1.0f / (float)a->cols,
                 {nullptr, a->d_amax, a->d_bias_out, ctx->d_status, FP8_E4, a->conv, a->margin}};
    if (a->d_amax || a->d_bias_out) p.sink.slot = take_slot(ctx);
    cudaStream_t st = (cudaStream_t)stream;
    if (a->dt == FP8_BF16) launch_fwd<FP8_BF16>(ctx, p, two, st);
    else if (a->dt == FP8_F16) launch_fwd<FP8_F16>(ctx, p, two, st);
    else launch_fwd<FP8_F32>(ctx, p, two, st);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

fp8_status_t fp8_norm_bwd(fp8_ctx *ctx, const fp8_norm_bwd_t *a, void *stream)
{
    using namespace fp8lin;
    if (!ctx || !a || !a->dy || !a->h || !a->d_rstd || (!a->dx && !a->dw && !a->db) || (a->d_amax && !a->dx)) return FP8_ERR_NULL;
    if (a->kind < 0 || a->kind > 1 || a->dt < 0 || a->dt > 2 || a->w_dt < 0 || a->w_dt > 2) return FP8_ERR_DTYPE;
    if (a->kind == FP8_NORM_LAYER && !a->d_mean) return FP8_ERR_NULL;
    if ((a->weight || a->dw || a->db) && a->w_dt != a->dt && a->w_dt != FP8_F32) return FP8_ERR_UNSUPPORTED;
    if (a->rows <= 0 || a->cols <= 0 || a->cols > kMaxCols) return FP8_ERR_SHAPE;
    if ((a->dw || a->db) && a->cols > (int64_t)1 << 22) return FP8_ERR_SHAPE;
    if (a->ld_dy < a->cols || a->ld_h < a->cols || (a->dh && a->ld_dh < a->cols) || (a->dx && a->ld_dx < a->cols)) return FP8_ERR_SHAPE;
    if (!element_aligned(a->dy, a->dt) || !element_aligned(a->h, a->dt) || !element_aligned(a->dh, a->dt) || !element_aligned(a->dx, a->dt) ||
        !element_aligned(a->weight, a->w_dt) || !element_aligned(a->dw, a->w_dt) || !element_aligned(a->db, a->w_dt) ||
        !element_aligned(a->d_mean, FP8_F32) || !element_aligned(a->d_rstd, FP8_F32) || !element_aligned(a->d_amax, FP8_F32))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    cudaStream_t st = (cudaStream_t)stream;
    unsigned grid = blocks_for_rows(ctx, a->rows, 4);
    const int sums = (a->dw ? 1 : 0) + (a->db ? 1 : 0);
    if (sums) {
        const int64_t lines = (int64_t)(ctx->partial_bytes / sizeof(float)) / (sums * a->cols);   // at least two (cols up to 2^22)
        if (grid > lines) grid = (unsigned)lines;
    }
    NormBwd p = {a->dy, a->h, a->dh, a->weight, a->d_mean, a->d_rstd, a->dx, nullptr, nullptr, a->rows, a->ld_dy, a->ld_h, a->ld_dh,
                 a->ld_dx, (int)a->cols, a->w_dt, a->kind == FP8_NORM_LAYER, 1.0f / (float)a->cols,
                 {nullptr, a->d_amax, nullptr, ctx->d_status, FP8_E5, 0, 0}};
    if (a->d_amax) p.sink.slot = take_slot(ctx);
    if (a->dw) p.part_w = ctx->d_partial;
    if (a->db) p.part_b = ctx->d_partial + (a->dw ? (int64_t)grid * a->cols : 0);
    if (a->dt == FP8_BF16) launch_bwd<FP8_BF16>(ctx, p, grid, st);
    else if (a->dt == FP8_F16) launch_bwd<FP8_F16>(ctx, p, grid, st);
    else launch_bwd<FP8_F32>(ctx, p, grid, st);
    if (cudaGetLastError() != cudaSuccess) return FP8_ERR_CUDA;
    if (sums) {
        count_launch();
        norm_bwd_sum_kernel<<<dim3((unsigned)((a->cols + 31) / 32), 2), 256, 0, st>>>(p.part_w, p.part_b, (int)grid, (int)a->cols, a->w_dt,
                                                                                   a->dw, a->db);
    }
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

}  // extern "C"
