// Layer norm and its root-mean-square form, forward (with the residual sum, and the E4 bytes and amax of the output) and
// backward.
#include <algorithm>

#include "fp8_norm.h"
#include "kv_common.cuh"
#include "ptx.cuh"
#include "row_common.cuh"

namespace fp8lin {

constexpr int kMaxCols = 1 << 30;

struct NormFwd {
    const void *x, *res, *w, *b;
    void *h, *y;
    float *mean, *rstd;
    uint8_t *y8;
    const int32_t *bias;   // of y8: given, or what the first pass left
    int64_t rows, ld_x, ld_res, ld_h, ld_y;
    int cols, w_dt, delta, layer;
    double inv_cols;   // (averages are one product of 64 bits: an FP32 reciprocal would be off for all rows alike)
    float eps;
    AmaxSink sink;
};

__device__ __forceinline__ float average(float sum, double inv_cols) { return (float)((double)sum * inv_cols); }
// Mean and sum of squared deviations of a row from its first estimate of the mean and the sums {d, d^2} of the deviations
// from that.  The estimate carries the rounding of a sum of whole numbers; where the mean is far above the spread (eight times,
// say), the mean of the small deviations corrects it, which is what keeps the spread's digits.
__device__ __forceinline__ float2 corrected(float estimate, float2 sums, int cols, double inv_cols)
{
    if (estimate * estimate <= 64.0f * average(sums.y, inv_cols)) return make_float2(estimate, sums.y);
    const float mean = estimate + average(sums.x, inv_cols), e = mean - estimate;
    const float squares = __fmaf_rn(-e, __fmaf_rn(-(float)cols, e, 2.0f * sums.x), sums.y);
    return make_float2(mean, squares < 0.0f ? 0.0f : squares);   // (NaN stays)
}

__device__ __forceinline__ float variance(float squares, double inv_cols, float eps) { return (float)((double)squares * inv_cols + (double)eps); }
// Squares that FP32 holds, with their digits.  Where they pass it, or come near its subnormal numbers, a row's statistics are taken
// again from its deviations times a power of two (2^-96, 2^96), which is exact for all that count: a row of any finite size is
// normalised.  (Of small squares the mean is good; of large ones it is taken again too.  NaN goes the same way and comes back.)
constexpr float kLeastVariance = 0x1p-90f, kFarDown = 0x1p-96f, kFarUp = 0x1p96f;
__device__ __forceinline__ bool held_by_fp32(float variance)   // (from kLeastVariance to FLT_MAX: one comparison of the bits)
{
    return __builtin_expect(__float_as_uint(variance) - __float_as_uint(kLeastVariance) <= __float_as_uint(FLT_MAX) - __float_as_uint(kLeastVariance), 1);
}
__device__ __forceinline__ float far_factor(float rstd) { return rstd >= 0x1p45f ? kFarUp : kFarDown; }   // (rstd: of such a variance)
// The estimate of the mean to go on from; `sum`: of the row times 2^-96.
__device__ __forceinline__ float far_estimate(float by, float estimate, float sum, double inv_cols)
{
    return by == kFarUp ? estimate : average(sum, inv_cols) * kFarUp;
}
// `corrected` of sums over deviations times `by`; the estimate and the mean are as they are.
__device__ __forceinline__ float2 corrected_far(float by, float estimate, float2 sums, int cols, double inv_cols)
{
    const float scaled = estimate * by;
    if (scaled * scaled <= 64.0f * average(sums.y, inv_cols)) return make_float2(estimate, sums.y);
    const float mean = estimate + average(sums.x, inv_cols) * (by == kFarUp ? kFarDown : kFarUp), e = (mean - estimate) * by;
    const float squares = __fmaf_rn(-e, __fmaf_rn(-(float)cols, e, 2.0f * sums.x), sums.y);
    return make_float2(mean, squares < 0.0f ? 0.0f : squares);
}
// 1 / standard deviation from a sum of squared deviations times `by`.
__device__ __forceinline__ float far_inverse(float by, float squares, double inv_cols, float eps)
{
    const double back = 1.0 / (double)by, var = (double)squares * inv_cols * back * back + (double)eps;
    const float f = var < (double)kLeastVariance ? kFarUp : var > (double)FLT_MAX ? kFarDown : 1.0f;
    return __frsqrt_rn((float)(var * (double)f * (double)f)) * f;
}

template <int DT>
__device__ __forceinline__ float normalised(float h, float mean, float rstd, float w, float b)
{
    return element_value<DT>(element_bits<DT>(__fmaf_rn(__fmul_rn(__fsub_rn(h, mean), rstd), w, b)));
}
__device__ __forceinline__ float weight_at(const void *w, int w_dt, int j) { return w ? load_any(w, w_dt, j) : 1.0f; }
__device__ __forceinline__ float shift_at(const void *b, int w_dt, int j) { return b ? load_any(b, w_dt, j) : 0.0f; }

// The launch behind may start when no block of this one waits for a place any more; it waits for this one's end itself.
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Any sizes and alignment, element by element: T threads a row.  HELD > 0: a thread holds that many elements (T * HELD >= cols) and
// the row is read once; 0: any length, three walks over it.  CAST_ONLY: the statistics are there, bytes are wanted.  Bound by the
// chain of a row (loads, two sums, stores): 1531 x 1027 FP32 in 10.4 us from a graph, of which an empty launch is 4.3 (1.2 TB/s);
// 1098 x 969 BF16 with a residual 8.5, by three walks 10.5.
template <int DT, bool CAST_ONLY, int T, int HELD>
__global__ void __launch_bounds__(T, 1024 / T) norm_fwd_any_kernel(const NormFwd p)
{
    constexpr int kTurns = HELD ? HELD : 1;
    constexpr bool kAhead = HELD > 0 && HELD <= 8;   // the next row's elements are on their way while this one is reduced
    __shared__ float part[T / 32];
    __shared__ float2 part2[T / 32];
    uint32_t key = 0;
    bool sat = false;
    const bool bytes = p.y8 && p.bias;
    if (!CAST_ONLY) launch_next();
    // (up to eight of each, the coefficients too are held: they would be waited for behind each row's sums)
    constexpr bool kHoldCoefficients = HELD > 0 && HELD <= 8;
    float held_w[kTurns], held_b[kTurns];
    if (kHoldCoefficients) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int j = (int)threadIdx.x + i * T;
            held_w[i] = j < p.cols ? weight_at(p.w, p.w_dt, j) : 0.0f;
            held_b[i] = j < p.cols ? shift_at(p.b, p.w_dt, j) : 0.0f;
        }
    }
    if (CAST_ONLY) wait_for_launch_before();
    Pow2Pair scale = {1.0f, 1.0f};
    if (bytes) scale = make_pow2_pair(__ldcg(p.bias) + p.delta);
    const bool from_h = CAST_ONLY && p.h;
    float x[kTurns], res[kTurns];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int j = (int)threadIdx.x + i * T;
            x[i] = res[i] = 0.0f;
            if (j >= p.cols) continue;
            x[i] = from_h ? load1<DT>(p.h, r * p.ld_h + j) : load1<DT>(p.x, r * p.ld_x + j);
            if (p.res && !from_h) res[i] = load1<DT>(p.res, r * p.ld_res + j);
        }
    };
    if (kAhead && blockIdx.x < p.rows) fetch(blockIdx.x);
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        float held[kTurns];
        const int64_t next = r + gridDim.x;
        auto sum_at = [&](int j) {
            float v = load1<DT>(p.x, r * p.ld_x + j);
            if (p.res) v = element_value<DT>(element_bits<DT>(v + load1<DT>(p.res, r * p.ld_res + j)));
            return v;
        };
        // f(element, its column, its place), for all of the thread's
        auto each = [&](auto f) {
            if (HELD) {
#pragma unroll
                for (int i = 0; i < kTurns; ++i)
                    if ((int)threadIdx.x + i * T < p.cols) f(held[i], (int)threadIdx.x + i * T, i);
            } else {
                for (int j = threadIdx.x; j < p.cols; j += T) f(p.h ? load1<DT>(p.h, r * p.ld_h + j) : sum_at(j), j, 0);
            }
        };
        if (HELD) {
            if (!kAhead) fetch(r);
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                held[i] = x[i];
                if (p.res && !from_h) held[i] = element_value<DT>(element_bits<DT>(x[i] + res[i]));
            }
            if (kAhead && next < p.rows) fetch(next);
        }
        float mean = 0.0f, rstd;
        if (CAST_ONLY) {
            mean = p.layer ? __ldcg(p.mean + r) : 0.0f;
            rstd = __ldcg(p.rstd + r);
        } else {
            float s = 0.0f;
            if (!HELD && p.h)
                for (int j = threadIdx.x; j < p.cols; j += T) store_bits<DT>(p.h, r * p.ld_h + j, element_bits<DT>(sum_at(j)));
            each([&](float v, int j, int) {
                if (HELD && p.h) store_bits<DT>(p.h, r * p.ld_h + j, element_bits<DT>(v));
                s += v;
            });
            s = block_sum<T>(s, part);
            if (p.layer) mean = average(s, p.inv_cols);
            float2 q = make_float2(0.0f, 0.0f);
            each([&](float v, int, int) {
                const float d = v - mean;
                q = make_float2(q.x + d, __fmaf_rn(d, d, q.y));
            });
            q = block_sum2<T>(q, part2);
            if (p.layer) {
                q = corrected(mean, q, p.cols, p.inv_cols);
                mean = q.x;
            }
            const float var = variance(q.y, p.inv_cols, p.eps);
            rstd = __frsqrt_rn(var);
            if (!held_by_fp32(var)) {
                const float by = far_factor(rstd);
                s = 0.0f;
                each([&](float v, int, int) { s = __fmaf_rn(v, kFarDown, s); });
                s = block_sum<T>(s, part);
                if (p.layer) mean = far_estimate(by, mean, s, p.inv_cols);
                q = make_float2(0.0f, 0.0f);
                each([&](float v, int, int) {
                    const float d = (v - mean) * by;
                    q = make_float2(q.x + d, __fmaf_rn(d, d, q.y));
                });
                q = block_sum2<T>(q, part2);
                if (p.layer) {
                    q = corrected_far(by, mean, q, p.cols, p.inv_cols);
                    mean = q.x;
                }
                rstd = far_inverse(by, q.y, p.inv_cols, p.eps);
            }
            if (threadIdx.x == 0) {
                if (p.mean) p.mean[r] = mean;
                if (p.rstd) p.rstd[r] = rstd;
            }
        }
        if (p.y || bytes || p.sink.slot) {
            each([&](float h, int j, int i) {
                const float w = kHoldCoefficients ? held_w[i] : weight_at(p.w, p.w_dt, j);
                const float b = kHoldCoefficients ? held_b[i] : shift_at(p.b, p.w_dt, j);
                const float v = normalised<DT>(h, mean, rstd, w, b);
                key = max(key, magnitude_key(v));
                if (p.y && !CAST_ONLY) store_bits<DT>(p.y, r * p.ld_y + j, element_bits<DT>(v));
                if (bytes) {
                    const float z = v * scale.first * scale.second;
                    sat = sat || clips<FP8_E4>(z);
                    p.y8[r * p.cols + j] = (uint8_t)(cvt_pair<FP8_E4>(0.0f, z) & 0xFFu);
                }
            });
        }
    }
    if (sat) raise_flags(p.sink.d_status, FP8_FLAG_SATURATED);
    if (!CAST_ONLY) sink_amax(key, p.sink);
}

// ---------------------------------------------------------------------------------------------------------------------
// rows of whole 16-byte vectors
// ---------------------------------------------------------------------------------------------------------------------
// TPR threads hold a row in registers, EPT elements each (TPR * EPT >= cols): the statistics, the output and its bytes come
// from one reading.
template <int DT>
constexpr int kPerVec = DT == FP8_F32 ? 4 : 8;
template <int TPR>
constexpr int kRowBlock = TPR < 128 ? 128 : TPR;   // threads of a block: four rows at a time where a warp holds one
// Blocks of the forward kernels that an SM's registers hold at once, which their grids are made of (as far as shared memory
// allows): each walks its share of the rows, and a block more than that would walk its share alone at the end.
template <int TPR, int EPT>
constexpr int kResident = TPR == 32 ? (EPT == 8 ? 8 : EPT == 16 ? 6 : 4) : TPR == 128 ? (EPT == 16 ? 6 : 4) : TPR == 256 ? 2 : 1;
// Groups of TPR threads of the backward kernel's block, of which an SM has one: the sums of its rows leave it as one line.
template <int TPR, int EPT>
constexpr int kSumGroups = TPR == 32 ? (EPT == 8 ? 24 : EPT == 16 ? 16 : 12) : TPR == 128 ? (EPT == 16 ? 5 : 3) : TPR == 256 ? 2 : 1;
constexpr int kMostGroups = 24;

// The rows that a group of TPR threads walks, on their way into shared memory `depth` rows ahead: bulk copies that one thread
// starts.  Neither registers nor a barrier wait for the memory, and a row's 32 elements a thread leave time for little else.
constexpr int kMostAhead = 4;
struct RowRing {
    uint64_t full[kMostGroups][kMostAhead];
    int abort_flag;
};
struct RowSource {
    const uint8_t *base[3];   // rows, NULL for one that is not there
    int64_t stride[3];        // in bytes
    uint32_t row_bytes;
    int inputs;               // of the three, those that are there
};
template <int TPR>
struct RowWalk {
    const RowSource &src;
    RowRing &ring;
    uint8_t *slots;           // this group's
    uint32_t slot_bytes;
    int depth, group;
    unsigned *d_status;
    bool in_time = true;      // no wait of this thread's has run out
    __device__ __forceinline__ RowWalk(const RowSource &s, RowRing &r, uint8_t *smem, int ahead, unsigned *status)
        : src(s), ring(r), slot_bytes(s.row_bytes * s.inputs), depth(ahead), group(threadIdx.x / TPR), d_status(status)
    {
        slots = smem + (uint64_t)group * depth * slot_bytes;
        if (threadIdx.x == 0) {
            for (int g = 0; g < (int)blockDim.x / TPR; ++g)
                for (int i = 0; i < kMostAhead; ++i) mbar_init(smem_u32(&ring.full[g][i]), 1);
            ring.abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
    }
    // one thread of the group: row r into slot s (none any more behind a wait that ran out)
    __device__ __forceinline__ void start(int64_t r, int s) const
    {
        if (!in_time) return;
        const uint64_t once = l2_policy_evict_first();   // (what is written stays in L2 for the launch behind)
        const uint32_t bar = smem_u32(&ring.full[group][s]);
        uint32_t to = smem_u32(slots + s * slot_bytes);
        mbar_expect_tx(bar, slot_bytes);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (!src.base[i]) continue;
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(to),
                         "l"(src.base[i] + r * src.stride[i]), "r"(src.row_bytes), "r"(bar), "l"(once)
                         : "memory");
            to += src.row_bytes;
        }
    }
    // (a wait that runs out raises the flag; the walk goes on with what is there, without waiting again)
    __device__ __forceinline__ const uint4 *wait(int s, uint32_t parity)
    {
        in_time = mbar_wait(smem_u32(&ring.full[group][s]), parity, &ring.abort_flag, d_status) && in_time;
        return reinterpret_cast<const uint4 *>(slots + s * slot_bytes);
    }
    // the block's shared memory is given up only when copies on their way have had time to arrive
    __device__ __forceinline__ void finish() const
    {
        if (*reinterpret_cast<volatile int *>(&ring.abort_flag)) __nanosleep(1000000);
    }
};

// A vector's coefficients from column col on (16-byte loads), `fill` where there are none.
template <int DT, bool WF32>
__device__ __forceinline__ void load_coefficients(const void *w, int col, float fill, Pair (&f)[kVecPairs<DT>])
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < kVecPairs<DT>; ++i) f[i] = pair_of(fill);
    } else if (WF32) {
#pragma unroll
        for (int i = 0; i < kVecPairs<DT>; i += 2) {
            const float4 v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(w) + col + 2 * i));
            f[i] = make_pair(v.x, v.y);
            f[i + 1] = make_pair(v.z, v.w);
        }
    } else {
        unpack_pairs<DT>(__ldg(reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(w) + (int64_t)col * InType<DT>::kBytes)), f);
    }
}

// Coefficients of a thread's own vectors: of the tensors' type they are held packed, FP32 ones are read again for each row.
template <int DT, bool WF32, int VECS>
struct HeldCoefficients {
    uint4 raw[WF32 ? 1 : VECS];
    const void *source;
    float fill;
    __device__ __forceinline__ HeldCoefficients(const void *w, float f, int t, int threads, int row_vecs) : source(w), fill(f)
    {
        if (WF32) return;
        const uint32_t one = DT == FP8_F32 ? 0x3F800000u : DT == FP8_BF16 ? 0x3F803F80u : 0x3C003C00u, all = f == 1.0f ? one : 0u;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            raw[WF32 ? 0 : i] = make_uint4(all, all, all, all);
            if (w && t + i * threads < row_vecs) raw[WF32 ? 0 : i] = __ldg(reinterpret_cast<const uint4 *>(w) + t + i * threads);
        }
    }
    // of vector i, whose first column is col
    __device__ __forceinline__ void get(int i, int col, Pair (&f)[kVecPairs<DT>]) const
    {
        if (WF32) load_coefficients<DT, WF32>(source, col, fill, f);
        else unpack_pairs<DT>(raw[WF32 ? 0 : i], f);
    }
};

// y of a vector, rounded to the tensors' type (the operations of `normalised`, in their order)
template <int DT>
__device__ __forceinline__ uint4 normalise_vector(const Pair (&h)[kVecPairs<DT>], float mean, float rstd, const Pair (&w)[kVecPairs<DT>],
                                                  const Pair (&b)[kVecPairs<DT>])
{
    const Pair less = pair_of(-mean), by = pair_of(rstd);
    Pair v[kVecPairs<DT>];
#pragma unroll
    for (int i = 0; i < kVecPairs<DT>; ++i) v[i] = fma((h[i] + less) * by, w[i], b[i]);
    return pack_pairs<DT>(v);
}
// h of a vector: x, or x + residual rounded to the type.
template <int DT>
__device__ __forceinline__ void sum_vector(const uint4 &x, const uint4 &res, Pair (&h)[kVecPairs<DT>], uint4 &packed)
{
    Pair f[kVecPairs<DT>];
    unpack_pairs<DT>(x, h);
    unpack_pairs<DT>(res, f);
#pragma unroll
    for (int i = 0; i < kVecPairs<DT>; ++i) h[i] = h[i] + f[i];
    packed = pack_pairs<DT>(h);
    unpack_pairs<DT>(packed, h);
}

// E4 bytes under one bias; `peak`: the largest magnitudes of y so far (packed), which say whether one was clipped.
struct ByteScale {
    float first, second;
    bool two;   // (uniform: biases beyond what one FP32 power of two holds)
    __device__ __forceinline__ explicit ByteScale(int shift)
    {
        const Pow2Pair p = make_pow2_pair(shift);
        first = p.first;
        second = p.second;
        two = second != 1.0f;
    }
    __device__ __forceinline__ float of(float y) const { return y * first * second; }
    // to y8 + at (8 or 4 bytes, aligned)
    template <int DT>
    __device__ __forceinline__ void store(uint8_t *y8, int64_t at, const uint4 &y, uint32_t &peak) const
    {
        const uint32_t words[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) peak = max_packed<DT>(peak, words[i] & (DT == FP8_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu));
        Pair v[kVecPairs<DT>];
        uint32_t pairs[4] = {};
        unpack_pairs<DT>(y, v);
        if (two)
#pragma unroll
            for (int i = 0; i < kVecPairs<DT>; ++i) v[i] = v[i] * pair_of(second);
#pragma unroll
        for (int i = 0; i < kVecPairs<DT>; ++i) {
            float lo, hi;
            split(v[i] * pair_of(first), lo, hi);
            pairs[i] = cvt_pair<FP8_E4>(hi, lo);
        }
        if (DT == FP8_F32) __stcs(reinterpret_cast<uint32_t *>(y8 + at), pairs[0] | (pairs[1] << 16));
        else __stcs(reinterpret_cast<uint2 *>(y8 + at), make_uint2(pairs[0] | (pairs[1] << 16), pairs[2] | (pairs[3] << 16)));
    }
    template <int DT>
    __device__ __forceinline__ bool clipped(uint32_t peak) const { return clips<FP8_E4>(of(packed_top<DT>(peak))); }
};

// From a row's elements and an estimate of its mean: sums of deviations (FAR: times `by`) and of their squares.  `left`: row_vecs - t.
template <int TPR, bool FAR, int VECS, int PAIRS>
__device__ __forceinline__ float2 row_deviations(const Pair (&h)[VECS][PAIRS], int left, float mean, float by, float2 *part)
{
    const Pair less = pair_of(-mean), by2 = pair_of(by);
    Pair d1 = pair_of(0.0f), d2 = d1;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        if (i * TPR >= left) continue;
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) {
            Pair d = h[i][k] + less;
            if (FAR) d = d * by2;
            d1 = d1 + d;
            d2 = fma(d, d, d2);
        }
    }
    return block_sum2<TPR>(make_float2(sum_of(d1), sum_of(d2)), part);
}
// Mean and 1 / standard deviation; false where they are to be taken again.
template <int TPR, int VECS, int PAIRS>
__device__ __forceinline__ bool row_statistics(const NormFwd &p, const Pair (&h)[VECS][PAIRS], int left, float &mean, float &rstd, float2 *part2)
{
    float2 q = row_deviations<TPR, false>(h, left, mean, 1.0f, part2);
    if (p.layer) {
        q = corrected(mean, q, p.cols, p.inv_cols);
        mean = q.x;
    }
    const float var = variance(q.y, p.inv_cols, p.eps);
    rstd = __frsqrt_rn(var);
    return held_by_fp32(var);
}
// (behind row_statistics; shared memory is used in the same order, a barrier lies between two uses of a word)
template <int TPR, int VECS, int PAIRS>
__device__ __forceinline__ void far_row_statistics(const NormFwd &p, const Pair (&h)[VECS][PAIRS], int left, float &mean, float &rstd, float *part,
                                                   float2 *part2)
{
    const float by = far_factor(rstd);
    const Pair down = pair_of(kFarDown);
    Pair s = pair_of(0.0f);
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        if (i * TPR >= left) continue;
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) s = fma(h[i][k], down, s);
    }
    const float sum = block_sum<TPR>(sum_of(s), part);
    if (p.layer) mean = far_estimate(by, mean, sum, p.inv_cols);
    float2 q = row_deviations<TPR, true>(h, left, mean, by, part2);
    if (p.layer) {
        q = corrected_far(by, mean, q, p.cols, p.inv_cols);
        mean = q.x;
    }
    rstd = far_inverse(by, q.y, p.inv_cols, p.eps);
}

// Few rows whose bytes are wanted: the blocks are one cluster that knows the amax when its rows are done, and casts them from
// shared memory in the same launch.  Bound by the chain of one row (6.2 us from a graph for one row of 8192 BF16 with a residual,
// an empty launch is 4.3); from the third row of a block on two launches are quicker (549 x 128: 22 us so, 8.4 in two).
template <int DT, bool WF32, int TPR, int EPT>
__global__ void __launch_bounds__(kRowBlock<TPR>) norm_fwd_cluster_kernel(const NormFwd p)
{
    constexpr int kN = kPerVec<DT>, kPairs = kVecPairs<DT>, kVecs = EPT / kN, kSize = InType<DT>::kBytes, kGroups = kRowBlock<TPR> / TPR;
    extern __shared__ __align__(16) uint4 stage[];   // y of this block's rows
    __shared__ float part[TPR / 32];
    __shared__ float2 part2[2][TPR / 32];
    __shared__ uint32_t block_key;
    int turn = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int64_t first = (int64_t)blockIdx.x * kGroups + group, step = (int64_t)gridDim.x * kGroups;
    const int row_vecs = p.cols / kN;
    uint32_t acc = 0;
    if (threadIdx.x == 0) block_key = 0u;
    const HeldCoefficients<DT, WF32, kVecs> weight(p.w, 1.0f, t, TPR, row_vecs), shift(p.b, 0.0f, t, TPR, row_vecs);
    for (int64_t r = first; r < p.rows; r += step, turn ^= 1) {
        const uint4 *px = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.x) + r * p.ld_x * kSize);
        const uint4 *pr = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.res) + r * p.ld_res * kSize);
        uint4 *ph = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.h) + r * p.ld_h * kSize);
        Pair h[kVecs][kPairs], s = pair_of(0.0f);
        uint4 x[kVecs], res[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (t + i * TPR >= row_vecs) continue;
            x[i] = px[t + i * TPR];
            if (p.res) res[i] = pr[t + i * TPR];
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (t + i * TPR >= row_vecs) continue;
            if (p.res) sum_vector<DT>(x[i], res[i], h[i], x[i]);
            else unpack_pairs<DT>(x[i], h[i]);
            if (p.h) ph[t + i * TPR] = x[i];
#pragma unroll
            for (int k = 0; k < kPairs; ++k) s = s + h[i][k];
        }
        float mean = p.layer ? average(block_sum<TPR>(sum_of(s), part), p.inv_cols) : 0.0f, rstd;
        if (!row_statistics<TPR>(p, h, row_vecs - t, mean, rstd, part2[turn])) far_row_statistics<TPR>(p, h, row_vecs - t, mean, rstd, part, part2[turn]);
        if (t == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int v = t + i * TPR;
            if (v >= row_vecs) continue;
            Pair w[kPairs], b[kPairs];
            weight.get(i, v * kN, w);
            shift.get(i, v * kN, b);
            const uint4 y = normalise_vector<DT>(h[i], mean, rstd, w, b);
            acc = fold_vector<DT>(acc, y);
            if (p.y) reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.y) + r * p.ld_y * kSize)[v] = y;
            stage[((r - first) / gridDim.x + group) * row_vecs + v] = y;
        }
    }
    const unsigned blocks = gridDim.x;
    uint32_t key = __reduce_max_sync(0xFFFFFFFFu, folded_key<DT>(acc));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) atomicMax(&block_key, key);
    __syncthreads();
    key = block_key;
    if (blocks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (unsigned b = 0; b < blocks; ++b) {
            uint32_t remote, other;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(&block_key)), "r"(b));
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(other) : "r"(remote) : "memory");
            key = max(key, other);
        }
        // (no block leaves while another reads its word)
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    unsigned flags = 0;
    const int bias = bias_from_amax_bits(key, FP8_E4, p.sink.conv, p.sink.margin, &flags);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (p.sink.d_amax) *p.sink.d_amax = __uint_as_float(key);
        *p.sink.d_bias = bias;
        if (flags) raise_flags(p.sink.d_status, flags);
    }
    const ByteScale scale(bias + p.delta);
    uint32_t peak = 0;
    for (int64_t r = first; r < p.rows; r += step)
        for (int v = t; v < row_vecs; v += TPR)
            scale.store<DT>(p.y8, r * p.cols + v * kN, stage[((r - first) / gridDim.x + group) * row_vecs + v], peak);
    if (scale.clipped<DT>(peak)) raise_flags(p.sink.d_status, FP8_FLAG_SATURATED);
    __syncwarp();
    if (blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Any number of rows: one reading, whatever is asked for but bytes under a bias that the call itself finds.  A row's fixed cost
// (two sums over its threads, some 150 instructions a thread) wants many elements a thread: 8192 x 4096 BF16 with a residual,
// the sum stored and the amax taken, 201 MB, took 55 us at 16 elements a thread and takes 40 at 32 with the coefficients held
// (5.0 TB/s).  Now bound by the chain of a row in sixteen warps an SM (issue slots 56 % used, memory 77 % of a plain copy's rate).
// Coefficients in shared memory and six rows a block at once: 44 us; five blocks an SM: 44.
template <int DT, bool WF32, int TPR, int EPT>
__global__ void __launch_bounds__(kRowBlock<TPR>, kResident<TPR, EPT>) norm_fwd_rows_kernel(const NormFwd p, const RowSource src, int depth)
{
    constexpr int kN = kPerVec<DT>, kPairs = kVecPairs<DT>, kVecs = EPT / kN, kSize = InType<DT>::kBytes, kGroups = kRowBlock<TPR> / TPR;
    extern __shared__ __align__(16) uint8_t slots[];
    __shared__ RowRing ring;
    __shared__ float part[TPR / 32];
    __shared__ float2 part2[2][TPR / 32];
    launch_next();
    RowWalk<TPR> walk(src, ring, slots, depth, p.sink.d_status);
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const int row_vecs = p.cols / kN;
    uint32_t acc = 0, peak = 0, parity = 0;
    int slot = 0, turn = 0;
    const bool bytes = p.y8 && p.bias, want_y = p.y || bytes || p.sink.slot;
    const ByteScale scale(bytes ? *p.bias + p.delta : 0);
    const HeldCoefficients<DT, WF32, kVecs> weight(p.w, 1.0f, t, TPR, row_vecs), shift(p.b, 0.0f, t, TPR, row_vecs);
    auto write = [&](int64_t r, const Pair(&h)[kVecs][kPairs], float mean, float rstd, bool again) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int v = t + i * TPR;
            if (v >= row_vecs) continue;
            Pair w[kPairs], b[kPairs];
            if (again) {   // (the others are held for the loop's sake)
                asm volatile("" ::: "memory");
                load_coefficients<DT, WF32>(p.w, v * kN, 1.0f, w);
                load_coefficients<DT, WF32>(p.b, v * kN, 0.0f, b);
            } else {
                weight.get(i, v * kN, w);
                shift.get(i, v * kN, b);
            }
            const uint4 y = normalise_vector<DT>(h[i], mean, rstd, w, b);
            if (p.sink.slot) acc = fold_vector<DT>(acc, y);
            if (p.y) reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.y) + r * p.ld_y * kSize)[v] = y;
            if (bytes) scale.store<DT>(p.y8, r * p.cols + v * kN, y, peak);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * kGroups + group;
    int64_t r = first;
    bool far = false;
    if (t == 0)
        for (int i = 0; i < depth && r + i * step < p.rows; ++i) walk.start(r + i * step, i);
    for (; r < p.rows; r += step, turn ^= 1) {
        const uint4 *in = walk.wait(slot, parity);
        Pair h[kVecs][kPairs], s = pair_of(0.0f);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int v = t + i * TPR;
            if (v >= row_vecs) continue;
            uint4 x = in[v];
            if (p.res) sum_vector<DT>(x, in[row_vecs + v], h[i], x);
            else unpack_pairs<DT>(x, h[i]);
            if (p.h) reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.h) + r * p.ld_h * kSize)[v] = x;
#pragma unroll
            for (int k = 0; k < kPairs; ++k) s = s + h[i][k];
        }
        float mean = p.layer ? average(block_sum<TPR>(sum_of(s), part), p.inv_cols) : 0.0f, rstd;
        const bool held = row_statistics<TPR>(p, h, row_vecs - t, mean, rstd, part2[turn]);
        far = far || !held;
        // every thread has read its part of the slot (a barrier, or the warp's exchange, lies behind it)
        if (TPR == 32) __syncwarp();
        if (t == 0) {
            if (r + depth * step < p.rows) walk.start(r + depth * step, slot);
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        if (++slot == depth) {
            slot = 0;
            parity ^= 1u;
        }
        if (want_y && held) write(r, h, mean, rstd, false);
    }
    walk.finish();
    // rows with statistics that FP32 does not hold, if there were some: once more, from memory, behind the loop that the others
    // run in (there, their code made 8192 x 4096 with bytes 3 % slower)
    if (far) {
        for (r = first; r < p.rows; r += step, turn ^= 1) {
            const uint8_t *from = static_cast<const uint8_t *>(p.h ? p.h : p.x) + r * (p.h ? p.ld_h : p.ld_x) * kSize;
            const uint8_t *res = p.h ? nullptr : static_cast<const uint8_t *>(p.res);
            Pair h[kVecs][kPairs], s = pair_of(0.0f);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int v = t + i * TPR;
                if (v >= row_vecs) continue;
                uint4 x = reinterpret_cast<const uint4 *>(from)[v];
                if (res) sum_vector<DT>(x, reinterpret_cast<const uint4 *>(res + r * p.ld_res * kSize)[v], h[i], x);
                else unpack_pairs<DT>(x, h[i]);
#pragma unroll
                for (int k = 0; k < kPairs; ++k) s = s + h[i][k];
                asm volatile("" ::: "memory");   // (vector by vector: registers are short)
            }
            float mean = p.layer ? average(block_sum<TPR>(sum_of(s), part), p.inv_cols) : 0.0f, rstd;
            if (row_statistics<TPR>(p, h, row_vecs - t, mean, rstd, part2[turn])) continue;
            far_row_statistics<TPR>(p, h, row_vecs - t, mean, rstd, part, part2[turn]);
            if (t == 0) {
                if (p.mean) p.mean[r] = mean;
                if (p.rstd) p.rstd[r] = rstd;
            }
            if (want_y) write(r, h, mean, rstd, true);
        }
    }
    if (scale.clipped<DT>(peak)) raise_flags(p.sink.d_status, FP8_FLAG_SATURATED);
    sink_amax(folded_key<DT>(acc), p.sink);
}

// The bytes of y from the sums and the statistics of the launch before, under the bias that it left.  Last rows first: what the
// launch before wrote last is what L2 holds.  8192 x 4096, 100 MB: 22 us (4.5 TB/s, L2 flushed), bound like the launch before; a
// thread per vector column and eight rows, without copies ahead, took 28.
template <int DT, bool WF32, int TPR, int EPT>
__global__ void __launch_bounds__(kRowBlock<TPR>, kResident<TPR, EPT>) norm_cast_rows_kernel(const NormFwd p, const RowSource src, int depth)
{
    constexpr int kN = kPerVec<DT>, kPairs = kVecPairs<DT>, kVecs = EPT / kN, kGroups = kRowBlock<TPR> / TPR;
    extern __shared__ __align__(16) uint8_t slots[];
    __shared__ RowRing ring;
    RowWalk<TPR> walk(src, ring, slots, depth, p.sink.d_status);
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    const int row_vecs = p.cols / kN;
    const HeldCoefficients<DT, WF32, kVecs> weight(p.w, 1.0f, t, TPR, row_vecs), shift(p.b, 0.0f, t, TPR, row_vecs);
    wait_for_launch_before();
    int64_t r = p.rows - 1 - ((int64_t)blockIdx.x * kGroups + group);
    if (t == 0)
        for (int i = 0; i < depth && r - i * step >= 0; ++i) walk.start(r - i * step, i);
    const ByteScale scale(__ldcg(p.bias) + p.delta);
    uint32_t peak = 0, parity = 0;
    int slot = 0;
    float mean = 0.0f, rstd = 0.0f;
    auto statistics = [&](int64_t row) {
        mean = p.layer ? __ldcg(p.mean + row) : 0.0f;
        rstd = __ldcg(p.rstd + row);
    };
    if (r >= 0) statistics(r);
    for (bool behind = false; r >= 0; r -= step, behind = true) {
        const uint4 *in = walk.wait(slot, parity);
        // (all are done with the row before: its slot is free)
        if (TPR == 32) __syncwarp();
        else __syncthreads();
        if (t == 0 && behind && r - (depth - 1) * step >= 0) walk.start(r - (depth - 1) * step, slot == 0 ? depth - 1 : slot - 1);
        const float m = mean, s = rstd;
        if (r - step >= 0) statistics(r - step);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int v = t + i * TPR;
            if (v >= row_vecs) continue;
            Pair h[kPairs], w[kPairs], b[kPairs];
            uint4 x = in[v];
            if (src.inputs == 2) sum_vector<DT>(x, in[row_vecs + v], h, x);
            else unpack_pairs<DT>(x, h);
            weight.get(i, v * kN, w);
            shift.get(i, v * kN, b);
            scale.store<DT>(p.y8, r * p.cols + v * kN, normalise_vector<DT>(h, m, s, w, b), peak);
        }
        if (++slot == depth) {
            slot = 0;
            parity ^= 1u;
        }
    }
    walk.finish();
    if (scale.clipped<DT>(peak)) raise_flags(p.sink.d_status, FP8_FLAG_SATURATED);
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

// Any sizes and alignment, element by element: T threads a row at a time.  HELD > 0: a thread holds that many elements and the
// sums of their columns; 0: any length, the sums of a block's rows grow in its own line of the workspace.
template <int DT, int T, int HELD>
__global__ void __launch_bounds__(T, 1024 / T) norm_bwd_any_kernel(const NormBwd p)
{
    constexpr int kTurns = HELD ? HELD : 1;
    __shared__ float2 part[2][T / 32];
    uint32_t key = 0;
    int turn = 0;
    float *pw = p.part_w ? p.part_w + (int64_t)blockIdx.x * p.cols : nullptr;
    float *pb = p.part_b ? p.part_b + (int64_t)blockIdx.x * p.cols : nullptr;
    float sum_w[kTurns], sum_b[kTurns], held_dy[kTurns], held_h[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) sum_w[i] = sum_b[i] = 0.0f;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn ^= 1) {
        const bool first = r == blockIdx.x;
        // f(dy, h, column, place), for all of the thread's
        auto each = [&](auto f) {
            if (HELD) {
#pragma unroll
                for (int i = 0; i < kTurns; ++i)
                    if ((int)threadIdx.x + i * T < p.cols) f(held_dy[i], held_h[i], (int)threadIdx.x + i * T, i);
            } else {
                for (int j = threadIdx.x; j < p.cols; j += T) f(load1<DT>(p.dy, r * p.ld_dy + j), load1<DT>(p.h, r * p.ld_h + j), j, 0);
            }
        };
        if (HELD) {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const int j = (int)threadIdx.x + i * T;
                if (j >= p.cols) continue;
                held_dy[i] = load1<DT>(p.dy, r * p.ld_dy + j);
                held_h[i] = load1<DT>(p.h, r * p.ld_h + j);
            }
        }
        const float mean = p.layer ? p.mean[r] : 0.0f, rstd = p.rstd[r];
        float2 s = make_float2(0.0f, 0.0f);
        each([&](float dy, float h, int j, int i) {
            const float xh = (h - mean) * rstd, g = p.w ? dy * load_any(p.w, p.w_dt, j) : dy;
            s = make_float2(s.x + g, __fmaf_rn(g, xh, s.y));
            if (HELD) {
                sum_w[i] = __fmaf_rn(dy, xh, sum_w[i]);
                sum_b[i] += dy;
            } else {
                if (pw) pw[j] = __fmaf_rn(dy, xh, first ? 0.0f : pw[j]);
                if (pb) pb[j] = first ? dy : pb[j] + dy;
            }
        });
        if (!p.dx) continue;
        s = block_sum2<T>(s, part[turn]);
        const float c1 = p.layer ? s.x * p.inv_cols : 0.0f, c2 = s.y * p.inv_cols;
        each([&](float dy, float h, int j, int) {
            const float xh = (h - mean) * rstd, g = p.w ? dy * load_any(p.w, p.w_dt, j) : dy;
            float v = rstd * (g - c1 - xh * c2);
            if (p.dh) v += load1<DT>(p.dh, r * p.ld_dh + j);
            const uint32_t bits = element_bits<DT>(v);
            key = max(key, magnitude_key(element_value<DT>(bits)));
            store_bits<DT>(p.dx, r * p.ld_dx + j, bits);
        });
    }
    if (HELD) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int j = (int)threadIdx.x + i * T;
            if (j >= p.cols) continue;
            if (pw) pw[j] = sum_w[i];
            if (pb) pb[j] = sum_b[i];
        }
    }
    sink_amax(key, p.sink);
}

// The same for rows of whole vectors: groups of TPR threads, each with rows of its own, for all of which a thread holds the sums of
// its columns: 64 registers at 32 elements, so rows wait in shared memory and are read from there twice.  8192 x 4096 BF16 with dh,
// 268 MB: 43 us (6.2 TB/s), bound by the memory; with rows in registers and 16 elements a thread 57.  A block an SM, because each
// block's sums are 32 KB that the launch behind has to read: with three it took 55 us in all, with one 52.
template <int DT, bool WF32, int TPR, int EPT>
__global__ void __launch_bounds__(kSumGroups<TPR, EPT> * TPR, 1) norm_bwd_rows_kernel(const NormBwd p, const RowSource src, int depth)
{
    constexpr int kN = kPerVec<DT>, kPairs = kVecPairs<DT>, kVecs = EPT / kN, kSize = InType<DT>::kBytes;
    extern __shared__ __align__(16) uint8_t slots[];
    __shared__ RowRing ring;
    __shared__ float2 part[kSumGroups<TPR, EPT>][2][TPR / 32];
    launch_next();
    RowWalk<TPR> walk(src, ring, slots, depth, p.sink.d_status);
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int groups = (int)blockDim.x / TPR;
    const int64_t step = (int64_t)gridDim.x * groups;
    const int row_vecs = p.cols / kN;
    uint32_t acc = 0, parity = 0;
    int slot = 0, turn = 0;
    Pair sum_w[kVecs][kPairs], sum_b[kVecs][kPairs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int k = 0; k < kPairs; ++k) sum_w[i][k] = sum_b[i][k] = pair_of(0.0f);
    const HeldCoefficients<DT, WF32, kVecs> weight(p.w, 1.0f, t, TPR, row_vecs);
    int64_t r = (int64_t)blockIdx.x * groups + group;
    if (t == 0)
        for (int i = 0; i < depth && r + i * step < p.rows; ++i) walk.start(r + i * step, i);
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto statistics = [&](int64_t row) {
        next_mean = p.layer ? p.mean[row] : 0.0f;
        next_rstd = p.rstd[row];
    };
    if (r < p.rows) statistics(r);
    for (bool behind = false; r < p.rows; r += step, turn ^= 1, behind = true) {
        const float mean = next_mean, rstd = next_rstd;
        if (r + step < p.rows) statistics(r + step);
        const uint4 *in = walk.wait(slot, parity);
        const Pair less = pair_of(-mean), by = pair_of(rstd);
        Pair p1 = pair_of(0.0f), p2 = p1;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            if (t + i * TPR >= row_vecs) continue;
            Pair y[kPairs], x[kPairs], w[kPairs];
            unpack_pairs<DT>(in[t + i * TPR], y);
            unpack_pairs<DT>(in[row_vecs + t + i * TPR], x);
            weight.get(i, (t + i * TPR) * kN, w);
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                const Pair xh = (x[k] + less) * by, g = y[k] * w[k];
                p1 = p1 + g;
                p2 = fma(g, xh, p2);
                sum_w[i][k] = fma(y[k], xh, sum_w[i][k]);
                sum_b[i][k] = sum_b[i][k] + y[k];
            }
        }
        const float2 s = group_sum2<TPR>(make_float2(sum_of(p1), sum_of(p2)), part[group][turn], group);
        // every thread is done with the row before (a barrier, or the warp's exchange, lies behind it): its slot is free
        if (TPR == 32) __syncwarp();
        if (t == 0 && behind && r + (depth - 1) * step < p.rows) walk.start(r + (depth - 1) * step, slot == 0 ? depth - 1 : slot - 1);
        if (p.dx) {
            const Pair c1 = pair_of(p.layer ? -s.x * p.inv_cols : 0.0f), c2 = pair_of(-s.y * p.inv_cols);
            uint4 *px = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.dx) + r * p.ld_dx * kSize);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int v = t + i * TPR;
                if (v >= row_vecs) continue;
                Pair y[kPairs], x[kPairs], w[kPairs];
                unpack_pairs<DT>(in[v], y);
                unpack_pairs<DT>(in[row_vecs + v], x);
                weight.get(i, v * kN, w);
#pragma unroll
                for (int k = 0; k < kPairs; ++k) y[k] = (fma((x[k] + less) * by, c2, y[k] * w[k]) + c1) * by;
                if (p.dh) {
                    unpack_pairs<DT>(in[2 * row_vecs + v], x);
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) y[k] = y[k] + x[k];
                }
                const uint4 out = pack_pairs<DT>(y);
                if (p.sink.slot) acc = fold_vector<DT>(acc, out);
                px[v] = out;
            }
        }
        if (++slot == depth) {
            slot = 0;
            parity ^= 1u;
        }
    }
    walk.finish();
    // the groups' sums meet where their rows were, and leave as one line
    float *lines = reinterpret_cast<float *>(slots);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *out = which ? p.part_b : p.part_w;
        if (!out) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int v = t + i * TPR;
            if (v >= row_vecs) continue;
#pragma unroll
            for (int k = 0; k < kN; k += 4) {
                float4 f;
                split(which ? sum_b[i][k / 2] : sum_w[i][k / 2], f.x, f.y);
                split(which ? sum_b[i][k / 2 + 1] : sum_w[i][k / 2 + 1], f.z, f.w);
                reinterpret_cast<float4 *>(lines + (int64_t)group * p.cols)[(v * kN + k) / 4] = f;
            }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < p.cols; j += (int)blockDim.x) {
            float s = lines[j];
            for (int g = 1; g < groups; ++g) s += lines[(int64_t)g * p.cols + j];
            out[(int64_t)blockIdx.x * p.cols + j] = s;
        }
    }
    sink_amax(folded_key<DT>(acc), p.sink);
}

// Sums of the blocks' lines, in one order: 32 columns a block, 32 lines at a time, eight of a thread's on their way.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) norm_bwd_sum_kernel(const float *part_w, const float *part_b, int lines, int cols, int w_dt,
                                                                   void *dw, void *db, int chunks)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const bool second = (int)blockIdx.x >= chunks;
    const int j = ((int)blockIdx.x - (second ? chunks : 0)) * 32 + lane;
    const float *part = (second ? part_b : part_w) + j;
    void *out = second ? db : dw;
    if (!out) return;
    wait_for_launch_before();
    float s = 0.0f;
    if (j < cols) {
        for (int i = group; i < lines; i += 8 * 32) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = i + k * 32 < lines ? __ldcg(part + (int64_t)(i + k * 32) * cols) : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
    }
    sums[group][lane] = s;
    __syncthreads();
    s = warp_sum(sums[lane][group]);
    const int column = j - lane + group;
    if (lane != 0 || column >= cols) return;
    if (w_dt == FP8_F32) store_bits<FP8_F32>(out, column, element_bits<FP8_F32>(s));
    else if (w_dt == FP8_BF16) store_bits<FP8_BF16>(out, column, element_bits<FP8_BF16>(s));
    else store_bits<FP8_F16>(out, column, element_bits<FP8_F16>(s));
}

// An output in an input's place lies as the input does.
static bool in_place(const void *out, int64_t ld_out, const void *in, int64_t ld_in, int64_t rows)
{
    return !out || out != in || rows == 1 || ld_out == ld_in;
}

static unsigned blocks_for_rows(const fp8_ctx *ctx, int64_t rows, int per_sm)
{
    const int64_t most = (int64_t)ctx->sm_count * per_sm;
    return (unsigned)(rows < most ? rows : most);
}

// Threads that hold a row, and elements that each of them holds.
template <int TPR, int EPT>
struct RowHold {
    static constexpr int kThreads = TPR, kElements = EPT;
};
constexpr int kMostHeld = 16384;
// A warp per row as long as 32 elements a lane hold it, then as few threads as that allow.  The forward kernels for rows of whole
// aligned vectors share the shapes, so that such a row's sums are taken in one order, however many rows there are and whether bytes are
// asked for or not.  (A call in which some tensor is not aligned goes to the kernel by elements.)
template <typename F>
static void by_row_shape(int cols, F f)
{
    if (cols <= 256) f(RowHold<32, 8>{});
    else if (cols <= 512) f(RowHold<32, 16>{});
    else if (cols <= 1024) f(RowHold<32, 32>{});
    else if (cols <= 2048) f(RowHold<128, 16>{});
    else if (cols <= 4096) f(RowHold<128, 32>{});
    else if (cols <= 8192) f(RowHold<256, 32>{});
    else f(RowHold<512, 32>{});
}
// Rows that are no whole vectors, or too long: threads, and elements that each of them holds (none: the row is walked).
template <typename F>
static void by_element_shape(int cols, F f)
{
    if (cols <= 512) f(RowHold<64, 8>{});
    else if (cols <= 1024) f(RowHold<128, 8>{});
    else if (cols <= 2048) f(RowHold<256, 8>{});
    else if (cols <= 4096) f(RowHold<512, 8>{});
    else if (cols <= 8192) f(RowHold<1024, 8>{});
    else if (cols <= 16384) f(RowHold<1024, 16>{});
    else f(RowHold<256, 0>{});
}

// Blocks an SM, and rows on their way for each group, that shared memory allows; false where not two rows fit.
static bool ring_size(int most_blocks, int groups, int64_t slot, int &blocks, int &depth)
{
    for (blocks = most_blocks; blocks > 0; --blocks) {
        const int64_t each = (227 << 10) / blocks - 4096 - (blocks > 1 ? 1024 : 0);   // (beside the fixed part)
        depth = (int)(each / (groups * slot));
        if (depth > kMostAhead) depth = kMostAhead;
        if (depth >= 2) return true;
    }
    return false;
}
constexpr int kRingBytes = (227 << 10) - 4096;

// Two passes as one launch of one cluster: up to eight blocks with two rows (or two times four) one after the other.
constexpr int kClusterBlocks = 8, kClusterRows = 2, kClusterStage = 96 << 10;

template <int DT, bool WF32>
static bool launch_fwd_cluster(const NormFwd &p, cudaStream_t st, cudaError_t &e)
{
    bool done = false;
    // (rows that the kernel for many of them does not take: theirs have to come from the same sums)
    int resident, depth;
    if (!ring_size(1, 1, (int64_t)p.cols * InType<DT>::kBytes * (p.res ? 2 : 1), resident, depth)) return false;
    by_row_shape(p.cols, [&](auto s) {
        constexpr int kThreads = decltype(s)::kThreads, kBlock = kRowBlock<kThreads>, kGroups = kBlock / kThreads;
        const int64_t blocks = (p.rows + kGroups - 1) / kGroups;
        int cluster = 1;
        while (cluster < kClusterBlocks && cluster < blocks) cluster *= 2;
        const int64_t each = (blocks + cluster - 1) / cluster, stage = each * kGroups * p.cols * InType<DT>::kBytes;
        if (each > kClusterRows || stage > kClusterStage) return;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)cluster);
        cfg.blockDim = dim3(kBlock);
        cfg.dynamicSmemBytes = (size_t)stage;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        count_launch();
        e = cudaLaunchKernelEx(&cfg, norm_fwd_cluster_kernel<DT, WF32, kThreads, decltype(s)::kElements>, p);
        done = true;
    });
    return done;
}

static RowSource row_source(int dt, int64_t cols, const void *a, int64_t ld_a, const void *b, int64_t ld_b, const void *c, int64_t ld_c)
{
    const int64_t size = dt == FP8_F32 ? 4 : 2;
    return RowSource{{static_cast<const uint8_t *>(a), static_cast<const uint8_t *>(b), static_cast<const uint8_t *>(c)},
                     {ld_a * size, ld_b * size, ld_c * size}, (uint32_t)(cols * size), 1 + (b ? 1 : 0) + (c ? 1 : 0)};
}

// One reading of all rows (two: and a second one for the bytes); false where the rows do not fit.
template <int DT, bool WF32>
static bool launch_fwd_rows(const fp8_ctx *ctx, const NormFwd &p, bool two, cudaStream_t st, cudaError_t &e)
{
    bool done = false;
    const RowSource src = row_source(DT, p.cols, p.x, p.ld_x, p.res, p.ld_res, nullptr, 0);
    by_row_shape(p.cols, [&](auto s) {
        constexpr int kThreads = decltype(s)::kThreads, kElements = decltype(s)::kElements, kBlock = kRowBlock<kThreads>, kGroups = kBlock / kThreads;
        const int64_t blocks = (p.rows + kGroups - 1) / kGroups;
        int resident, depth;
        auto grid = [&] { return (unsigned)std::min(blocks, (int64_t)ctx->sm_count * resident); };
        auto bytes = [&](const RowSource &from) { return (size_t)kGroups * depth * from.row_bytes * from.inputs; };
        if (!ring_size(kResident<kThreads, kElements>, kGroups, (int64_t)src.row_bytes * src.inputs, resident, depth)) return;
        NormFwd once = p;
        if (two) once.bias = nullptr;
        count_launch();
        norm_fwd_rows_kernel<DT, WF32, kThreads, kElements><<<grid(), kBlock, bytes(src), st>>>(once, src, depth);
        e = cudaGetLastError();
        done = true;
        if (!two || e != cudaSuccess) return;
        const RowSource sums = p.h ? row_source(DT, p.cols, p.h, p.ld_h, nullptr, 0, nullptr, 0) : src;
        ring_size(kResident<kThreads, kElements>, kGroups, (int64_t)sums.row_bytes * sums.inputs, resident, depth);
        e = launch_dependent_with(norm_cast_rows_kernel<DT, WF32, kThreads, kElements>, grid(), kBlock, bytes(sums), st, p, sums, depth);
    });
    return done;
}

template <int DT, bool WF32>
static cudaError_t allow_shared()
{
    cudaError_t e = cudaSuccess;
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    for (int cols : {256, 512, 1024, 2048, 4096, 8192, kMostHeld}) {
        by_row_shape(cols, [&](auto s) {
            if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_fwd_cluster_kernel<DT, WF32, decltype(s)::kThreads, decltype(s)::kElements>, attr, kClusterStage);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_fwd_rows_kernel<DT, WF32, decltype(s)::kThreads, decltype(s)::kElements>, attr, kRingBytes);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_cast_rows_kernel<DT, WF32, decltype(s)::kThreads, decltype(s)::kElements>, attr, kRingBytes);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(norm_bwd_rows_kernel<DT, WF32, decltype(s)::kThreads, decltype(s)::kElements>, attr, kRingBytes);
        });
    }
    return e;
}
cudaError_t configure_norm_kernels()
{
    cudaError_t e = allow_shared<FP8_BF16, false>();
    if (e == cudaSuccess) e = allow_shared<FP8_BF16, true>();
    if (e == cudaSuccess) e = allow_shared<FP8_F16, false>();
    if (e == cudaSuccess) e = allow_shared<FP8_F16, true>();
    return e == cudaSuccess ? allow_shared<FP8_F32, false>() : e;
}

// Whether every row, and every coefficient vector, consists of whole aligned vectors.
static bool whole_vectors(int dt, int64_t cols)
{
    return cols % (dt == FP8_F32 ? 4 : 8) == 0;
}
static bool fast_rows(const NormFwd &p, int dt)
{
    auto row = [&](const void *q, int64_t ld) { return !q || row_aligned(q, ld, dt, 16); };
    return whole_vectors(dt, p.cols) && p.cols <= kMostHeld && row(p.x, p.ld_x) && row(p.res, p.ld_res) && row(p.h, p.ld_h) && row(p.y, p.ld_y) &&
           row(p.w, 0) && row(p.b, 0) && (reinterpret_cast<uintptr_t>(p.y8) & 7u) == 0;
}

template <int DT, bool WF32>
static cudaError_t launch_fwd(const fp8_ctx *ctx, NormFwd p, bool two, cudaStream_t st)
{
    if (fast_rows(p, DT)) {
        cudaError_t e = cudaSuccess;
        if (two && launch_fwd_cluster<DT, WF32>(p, st, e)) return e;
        if (launch_fwd_rows<DT, WF32>(ctx, p, two, st, e)) return e;
    }
    NormFwd once = p;
    if (two) once.bias = nullptr;
    cudaError_t e = cudaSuccess;
    by_element_shape(p.cols, [&](auto s) {
        constexpr int kThreads = decltype(s)::kThreads, kElements = decltype(s)::kElements;
        const unsigned grid = blocks_for_rows(ctx, p.rows, 1024 / kThreads);
        count_launch();
        norm_fwd_any_kernel<DT, false, kThreads, kElements><<<grid, kThreads, 0, st>>>(once);
        e = cudaGetLastError();
        if (two && e == cudaSuccess) e = launch_dependent_with(norm_fwd_any_kernel<DT, true, kThreads, kElements>, grid, kThreads, 0, st, p);
    });
    return e;
}

// Lines of the workspace that a call's row sums take (as many blocks as its kernel has), within the workspace.
static unsigned bwd_blocks(const fp8_ctx *ctx, int64_t blocks, int per_sm, int sums, int64_t cols)
{
    int64_t n = (int64_t)ctx->sm_count * per_sm;
    if (n > blocks) n = blocks;
    if (sums) {
        const int64_t lines = (int64_t)(ctx->partial_bytes / sizeof(float)) / (sums * cols);   // at least two (cols up to 2^22)
        if (n > lines) n = lines;
    }
    return (unsigned)n;
}

template <int DT, bool WF32>
static unsigned launch_bwd(const fp8_ctx *ctx, NormBwd p, bool want_w, bool want_b, cudaStream_t st)
{
    auto row = [&](const void *q, int64_t ld) { return !q || row_aligned(q, ld, DT, 16); };
    const int sums = want_w || want_b ? 2 : 0;   // (one of the two alone takes the same blocks, and gives the same bits; dx needs no place)
    const bool fast = p.cols % kPerVec<DT> == 0 && p.cols <= kMostHeld && row(p.dy, p.ld_dy) && row(p.h, p.ld_h) && row(p.dh, p.ld_dh) &&
                      row(p.dx, p.ld_dx) && row(p.w, 0);
    unsigned grid = 0;
    auto lines = [&] {
        if (want_w) p.part_w = ctx->d_partial;
        if (want_b) p.part_b = ctx->d_partial + (int64_t)grid * p.cols;
    };
    bool done = false;
    const RowSource src = row_source(DT, p.cols, p.dy, p.ld_dy, p.h, p.ld_h, p.dh, p.ld_dh);
    if (fast)
        by_row_shape(p.cols, [&](auto s) {
            constexpr int kThreads = decltype(s)::kThreads, kElements = decltype(s)::kElements;
            // as many groups as have rows and two slots each
            const int64_t slot = (int64_t)src.row_bytes * src.inputs;
            int groups = (int)std::min((int64_t)kSumGroups<kThreads, kElements>, (p.rows + ctx->sm_count - 1) / ctx->sm_count), blocks, depth = 0;
            while (groups > 0 && !ring_size(1, groups, slot, blocks, depth)) --groups;
            if (groups == 0) return;
            grid = bwd_blocks(ctx, (p.rows + groups - 1) / groups, 1, sums, p.cols);
            lines();
            count_launch();
            norm_bwd_rows_kernel<DT, WF32, kThreads, kElements><<<grid, groups * kThreads, (size_t)groups * depth * slot, st>>>(p, src, depth);
            done = true;
        });
    if (!done) {
        by_element_shape(p.cols, [&](auto s) {
            constexpr int kThreads = decltype(s)::kThreads, kElements = decltype(s)::kElements;
            grid = bwd_blocks(ctx, p.rows, 1024 / kThreads, sums, p.cols);
            lines();
            count_launch();
            norm_bwd_any_kernel<DT, kThreads, kElements><<<grid, kThreads, 0, st>>>(p);
        });
    }
    return grid;
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
    if (!in_place(a->h, a->ld_h, a->x, a->ld_x, a->rows) || !in_place(a->h, a->ld_h, a->residual, a->ld_residual, a->rows)) return FP8_ERR_SHAPE;
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
                 a->kind == FP8_NORM_LAYER, 1.0 / (double)a->cols, a->eps,
                 {nullptr, a->d_amax, a->d_bias_out, ctx->d_status, FP8_E4, a->conv, a->margin}};
    if (a->d_amax || a->d_bias_out) p.sink.slot = take_slot(ctx);
    cudaStream_t st = (cudaStream_t)stream;
    const bool wide = a->w_dt == FP8_F32 && a->dt != FP8_F32;
    const cudaError_t e = a->dt == FP8_F32    ? launch_fwd<FP8_F32, false>(ctx, p, two, st)
                          : a->dt == FP8_BF16 ? (wide ? launch_fwd<FP8_BF16, true>(ctx, p, two, st) : launch_fwd<FP8_BF16, false>(ctx, p, two, st))
                          : wide              ? launch_fwd<FP8_F16, true>(ctx, p, two, st)
                                              : launch_fwd<FP8_F16, false>(ctx, p, two, st);
    return e == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
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
    if (!in_place(a->dx, a->ld_dx, a->dy, a->ld_dy, a->rows) || !in_place(a->dx, a->ld_dx, a->dh, a->ld_dh, a->rows)) return FP8_ERR_SHAPE;
    if (!element_aligned(a->dy, a->dt) || !element_aligned(a->h, a->dt) || !element_aligned(a->dh, a->dt) || !element_aligned(a->dx, a->dt) ||
        !element_aligned(a->weight, a->w_dt) || !element_aligned(a->dw, a->w_dt) || !element_aligned(a->db, a->w_dt) ||
        !element_aligned(a->d_mean, FP8_F32) || !element_aligned(a->d_rstd, FP8_F32) || !element_aligned(a->d_amax, FP8_F32))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    cudaStream_t st = (cudaStream_t)stream;
    NormBwd p = {a->dy, a->h, a->dh, a->weight, a->d_mean, a->d_rstd, a->dx, nullptr, nullptr, a->rows, a->ld_dy, a->ld_h, a->ld_dh,
                 a->ld_dx, (int)a->cols, a->w_dt, a->kind == FP8_NORM_LAYER, 1.0f / (float)a->cols,
                 {nullptr, a->d_amax, nullptr, ctx->d_status, FP8_E5, 0, 0}};
    if (a->d_amax) p.sink.slot = take_slot(ctx);
    const bool wide = a->w_dt == FP8_F32 && a->dt != FP8_F32, w = a->dw != nullptr, b = a->db != nullptr;
    const unsigned lines = a->dt == FP8_F32    ? launch_bwd<FP8_F32, false>(ctx, p, w, b, st)
                           : a->dt == FP8_BF16 ? (wide ? launch_bwd<FP8_BF16, true>(ctx, p, w, b, st) : launch_bwd<FP8_BF16, false>(ctx, p, w, b, st))
                           : wide              ? launch_bwd<FP8_F16, true>(ctx, p, w, b, st)
                                               : launch_bwd<FP8_F16, false>(ctx, p, w, b, st);
    if (cudaGetLastError() != cudaSuccess) return FP8_ERR_CUDA;
    if (w || b) {
        const int chunks = (int)((a->cols + 31) / 32);
        if (launch_dependent_with(norm_bwd_sum_kernel, 2u * chunks, kSumThreads, 0, st, ctx->d_partial, ctx->d_partial + (int64_t)lines * a->cols,
                             (int)lines, (int)a->cols, a->w_dt, a->dw, a->db, chunks) != cudaSuccess)
            return FP8_ERR_CUDA;
    }
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

}  // extern "C"
