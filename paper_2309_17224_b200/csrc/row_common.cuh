// What the row-wise kernels (norm.cu, loss.cu) share: elements of three types, reductions, the amax of an output.
#pragma once

#include <float.h>

#include "cast_common.cuh"

namespace fp8lin {

inline bool row_aligned(const void *p, int64_t ld, int dt, unsigned bytes)
{
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (dt == FP8_F32 ? 4 : 2))) & (bytes - 1)) == 0;
}
inline bool element_aligned(const void *p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (dt == FP8_F32 ? 3u : 1u)) == 0; }

// Launches go to the context's device, whichever is the caller's current one (the default streams of all devices share a
// handle).
struct OnDevice {
    int before = -1;
    explicit OnDevice(int device)
    {
        int now = device;
        if (cudaGetDevice(&now) == cudaSuccess && now != device && cudaSetDevice(device) == cudaSuccess) before = now;
    }
    ~OnDevice()
    {
        if (before >= 0) cudaSetDevice(before);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
};

// Where a call's amax goes (nowhere where slot is NULL): blocks fold their maxima into a slot of the context, the last
// one publishes the amax and, where asked, its scaling bias, and leaves the slot zeroed for the next call.
struct AmaxSink {
    unsigned *slot;
    float *d_amax;
    int32_t *d_bias;
    unsigned *d_status;
    int fmt, conv, margin;
};

#ifdef __CUDACC__

// v rounded to the tensors' type, as a float; the element's bits
template <int DT>
__device__ __forceinline__ uint32_t element_bits(float v)
{
    if (DT == FP8_F32) return __float_as_uint(v);
    uint32_t w;
    if (DT == FP8_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(0.0f), "f"(v));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(0.0f), "f"(v));
    return w & 0xFFFFu;
}
template <int DT>
__device__ __forceinline__ float element_value(uint32_t bits)
{
    if (DT == FP8_F32) return __uint_as_float(bits);
    if (DT == FP8_BF16) return __uint_as_float(bits << 16);
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)bits));
    return f;
}
template <int DT>
__device__ __forceinline__ void store_bits(void *y, int64_t i, uint32_t bits)
{
    if (DT == FP8_F32) reinterpret_cast<uint32_t *>(y)[i] = bits;
    else reinterpret_cast<uint16_t *>(y)[i] = (uint16_t)bits;
}
__device__ __forceinline__ float load_any(const void *x, int dt, int64_t i)
{
    if (dt == FP8_F32) return load1<FP8_F32>(x, i);
    return dt == FP8_BF16 ? load1<FP8_BF16>(x, i) : load1<FP8_F16>(x, i);
}

// A 16-byte vector's elements as floats.
template <int DT, int N>
__device__ __forceinline__ void unpack_vector(const uint4 &v, float (&f)[N])
{
    static_assert(N == (DT == FP8_F32 ? 4 : 8), "elements of 16 bytes");
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float g[4];
        unpack4<DT>(w + i / 4 * InType<DT>::kWords4, g);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[i + k] = g[k];
    }
}

// Two FP32 numbers an instruction (a register pair).
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair make_pair(float lo, float hi)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ Pair pair_of(float x) { return make_pair(x, x); }
__device__ __forceinline__ void split(Pair p, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.v)); }
__device__ __forceinline__ Pair operator+(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float sum_of(Pair p)
{
    float lo, hi;
    split(p, lo, hi);
    return lo + hi;
}

// Elements 2i, 2i + 1 of a 16-byte vector (FP32: of its four), and a vector of such pairs rounded to the type.
template <int DT>
constexpr int kVecPairs = DT == FP8_F32 ? 2 : 4;
template <int DT>
__device__ __forceinline__ void unpack_pairs(const uint4 &v, Pair (&f)[kVecPairs<DT>])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kVecPairs<DT>; ++i) {
        if (DT == FP8_F32) {
            f[i] = make_pair(__uint_as_float(w[2 * i % 4]), __uint_as_float(w[(2 * i + 1) % 4]));
        } else if (DT == FP8_BF16) {
            f[i] = make_pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        } else {
            float lo, hi;
            asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }" : "=f"(lo), "=f"(hi) : "r"(w[i]));
            f[i] = make_pair(lo, hi);
        }
    }
}
template <int DT>
__device__ __forceinline__ uint4 pack_pairs(const Pair (&f)[kVecPairs<DT>])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < kVecPairs<DT>; ++i) {
        float lo, hi;
        split(f[i], lo, hi);
        if (DT == FP8_F32) {
            w[2 * i % 4] = __float_as_uint(lo);
            w[(2 * i + 1) % 4] = __float_as_uint(hi);
        } else if (DT == FP8_BF16) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
        } else {
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(hi), "f"(lo));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The largest of packed elements; NaN is passed over.
template <int DT>
__device__ __forceinline__ uint32_t max_packed(uint32_t a, uint32_t b)
{
    uint32_t r;
    if (DT == FP8_F32) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    if (DT == FP8_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int DT>
__device__ __forceinline__ float packed_top(uint32_t a)
{
    return DT == FP8_F32 ? __uint_as_float(a) : fmaxf(element_value<DT>(a & 0xFFFFu), element_value<DT>(a >> 16));
}

// Largest magnitude of packed elements (as fp8_amax folds them), and its key.
template <int DT>
__device__ __forceinline__ uint32_t fold_vector(uint32_t acc, const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = DT == FP8_F32 ? max(acc, w[i] & 0x7FFFFFFFu) : __vmaxu2(acc, w[i] & 0x7FFF7FFFu);
    return acc;
}

// Magnitudes as unsigned numbers: NaN above infinity above what is finite.
__device__ __forceinline__ uint32_t magnitude_key(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int DT>
__device__ __forceinline__ uint32_t folded_key(uint32_t acc)
{
    if (DT == FP8_F32) return acc;
    return magnitude_key(element_value<DT>(max(acc & 0xFFFFu, acc >> 16)));
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sum over the block, to all threads.  `part`: one word a warp; two calls in a row use different words, and there is a
// barrier between a call and the one after the next.
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *part)
{
    v = warp_sum(v);
    if (THREADS == 32) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) v += part[i];
    return v;
}

template <int THREADS>
__device__ __forceinline__ float2 block_sum2(float2 v, float2 *part)
{
    v = make_float2(warp_sum(v.x), warp_sum(v.y));
    if (THREADS == 32) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) v = make_float2(v.x + part[i].x, v.y + part[i].y);
    return v;
}

// The same over a group of THREADS of a block with several groups (each has its own `part`, and barrier).
template <int THREADS>
__device__ __forceinline__ float2 group_sum2(float2 v, float2 *part, int group)
{
    v = make_float2(warp_sum(v.x), warp_sum(v.y));
    if (THREADS == 32) return v;
    const int warp = (threadIdx.x % THREADS) >> 5;
    if ((threadIdx.x & 31) == 0) part[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(THREADS) : "memory");
    v = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) v = make_float2(v.x + part[i].x, v.y + part[i].y);
    return v;
}

// Fold a thread's magnitude key into the sink; every thread of every block calls it once, at the end.
__device__ __forceinline__ void sink_amax(uint32_t key, const AmaxSink &o)
{
    __shared__ uint32_t warp_max[32];
    if (!o.slot) return;
    key = __reduce_max_sync(0xFFFFFFFFu, key);
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = key;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (unsigned i = 1; i < blockDim.x / 32; ++i) key = max(key, warp_max[i]);
    atomicMax(&o.slot[0], key);
    __threadfence();
    if (atomicAdd(&o.slot[1], 1u) + 1u != gridDim.x) return;
    __threadfence();
    key = atomicExch(&o.slot[0], 0u);
    o.slot[1] = 0u;
    if (o.d_amax) *o.d_amax = __uint_as_float(key);
    if (o.d_bias) {
        unsigned flags = 0;
        *o.d_bias = bias_from_amax_bits(key, o.fmt, o.conv, o.margin, &flags);
        if (flags) atomicOr(o.d_status, flags);
    }
}

#endif
}  // namespace fp8lin
