// Log probabilities of given tokens with entropy and top tokens, and the divergence from a teacher's listed tokens, each
// with the gradient of the logits.
#include <algorithm>

#include "fp8_loss.h"
#include "kv_common.cuh"
#include "row_common.cuh"

namespace fp8lin {

constexpr int kTopBuffer = 2048;     // candidates for the top tokens of a row
constexpr float kFloor = -200.0f;    // exponents (base 2) below it are zeros: 2^-200 is none of an FP32 sum
constexpr float kFarRest = -64.0f;   // ln of the unlisted tokens' sum (relative to the row's largest logit) that is good to 2^-16 of a share
constexpr float kLn2 = 0.693147180559945309f, kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the larger number, NaN if one is NaN (fmaxf drops it)
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// ---------------------------------------------------------------------------------------------------------------------
// a row, or a part of it, as head elements up to the first 16-byte boundary, whole vectors, tail elements
// ---------------------------------------------------------------------------------------------------------------------
template <int DT>
struct Row {
    static constexpr int kVec = DT == FP8_F32 ? 4 : 8;
    const uint8_t *base;
    int first, n, head, vecs, tail;   // first: element 0's place in the whole row;  tail: the first element behind the vectors
    __device__ __forceinline__ Row(const void *logits, int64_t at, int from, int count)
    {
        constexpr int kSize = InType<DT>::kBytes;
        base = static_cast<const uint8_t *>(logits) + (at + from) * kSize;
        first = from;
        n = count;
        head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15u)) & 15u) / kSize);
        vecs = (n - head) / kVec;
        tail = head + vecs * kVec;
    }
    __device__ __forceinline__ const uint4 *vectors() const { return reinterpret_cast<const uint4 *>(base + head * InType<DT>::kBytes); }
    __device__ __forceinline__ float at(int j) const { return load1<DT>(base, j); }
    // elements outside the vectors, at most one a thread (kVec - 1 on either side): its place, or -1
    __device__ __forceinline__ int edge(int t) const { return t < head ? t : tail + t - head < n ? tail + t - head : -1; }
};

// A vector whose elements are all -infinity.
template <int DT>
__device__ __forceinline__ uint4 no_vector()
{
    const uint32_t w = DT == FP8_F32 ? 0xFF800000u : DT == FP8_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
    return make_uint4(w, w, w, w);
}

// Orders like the numbers (-0 like 0); 0 is below every number's key.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ float warp_max(float x) { return order_value(__reduce_max_sync(0xFFFFFFFFu, order_key(x))); }

// Sums over exp(scale (x - m)): with d = c (x - m), c = scale * log2 e:  s = sum 2^d,  t = sum 2^d d.  While a row is read, m
// is not its largest number but one near it: it moves only when a term would pass 2^kLead, which most rows do once a thread
// (moving it costs an exponential and a branch that a whole warp takes when one lane does).
constexpr float kLead = 8.0f;
struct Sums {
    float m, s, t;
    // the same sums relative to another number
    __device__ __forceinline__ void relate(float to, float c)
    {
        const float d = fmaxf((m - to) * c, kFloor), f = exp2_approx(d);
        t = f * __fmaf_rn(d, s, t);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void lead(float x, float c)
    {
        if ((x - m) * c > kLead) relate(x, c);
    }
    __device__ __forceinline__ void join(Sums b, float c)
    {
        const float to = fmaxf(m, b.m);
        relate(to, c);
        b.relate(to, c);
        s += b.s;
        t += b.t;
    }
};
__device__ __forceinline__ Sums no_sums() { return Sums{-FLT_MAX, 0.0f, 0.0f}; }

// One element.
template <bool ENTROPY>
__device__ __forceinline__ void add_element(Sums &a, float x, float c)
{
    a.lead(x, c);
    const float d = max_nan((x - a.m) * c, kFloor), e = exp2_approx(d);
    a.s += e;
    if (ENTROPY) a.t = __fmaf_rn(e, d, a.t);
}

// Sums over the block relative to the largest number `top` of all threads, to all threads, always in the same order.  m is
// -infinity where there is no number.
template <int T>
struct JoinShared {
    float4 part[T / 32];
};
template <int T>
__device__ __forceinline__ Sums block_join(Sums a, float top, float c, JoinShared<T> &sh)
{
    const int lane = threadIdx.x & 31;
    a.relate(warp_max(a.m), c);
    a.s = warp_sum(a.s);
    a.t = warp_sum(a.t);
    top = warp_max(top);
    if (lane == 0) sh.part[threadIdx.x >> 5] = make_float4(a.m, a.s, a.t, top);
    __syncthreads();
    const float4 v = sh.part[lane % (T / 32)];
    a = Sums{v.x, v.y, v.z};
    a.relate(warp_max(a.m), c);
#pragma unroll
    for (int o = T / 64; o > 0; o >>= 1) {   // (each group of lanes holds all the parts)
        a.s += __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a.t += __shfl_xor_sync(0xFFFFFFFFu, a.t, o);
    }
    top = warp_max(v.w);
    if (a.s != 0.0f) a.relate(top, c);
    a.m = top;
    return a;
}

// ---------------------------------------------------------------------------------------------------------------------
// top tokens
// ---------------------------------------------------------------------------------------------------------------------
// larger logit first, then lower index
__device__ __forceinline__ unsigned long long top_key(float x, int j) { return ((unsigned long long)order_key(x) << 32) | (uint32_t)~j; }

template <int T>
struct TopShared {
    unsigned long long key[kTopBuffer], best[FP8_LOSS_TOP_MAX];
    uint32_t strip[T];
    int owner[T];   // strips that reach the bound
    int count, strips;
    uint32_t bound;
};

template <>
struct TopShared<64> {};   // 64 threads: a kernel without top tokens, so that shared memory holds as many blocks as registers

// The k largest of sh.key[0 .. n), in order, to sh.best.  Keys differ, so a key's place is the number of larger ones.
template <int T>
__device__ __forceinline__ void top_rank(TopShared<T> &sh, int n, int k)
{
    for (int at = threadIdx.x; at < n; at += T) {
        const unsigned long long mine = sh.key[at];
        int larger = 0;
        for (int o = 0; o < n; ++o) larger += sh.key[o] > mine;
        if (larger < k) sh.best[larger] = mine;
    }
    __syncthreads();
}

// The row's top k keys into sh.best.  m: the thread's own largest element (its strip: the vectors v = thread mod T, and its
// edge element).  A bound that k strips reach is reached by k elements; only those strips are read again.
template <int DT, int T>
__device__ __forceinline__ void find_top(const Row<DT> &row, float m, int k, TopShared<T> &sh)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int edge = row.edge(tid);
    // sixteen bits of the key are enough of a bound
    const uint32_t mine = tid < row.vecs || edge >= 0 ? order_key(m) >> 16 : 0u;
    sh.strip[tid] = mine;
    if (tid == 0) sh.count = sh.strips = 0;
    __syncthreads();
    if (tid < 32) {
        uint32_t own[T / 32], bound = 0;
#pragma unroll
        for (int i = 0; i < T / 32; ++i) own[i] = sh.strip[lane + 32 * i];
        for (int i = 0; k <= 8 && i < k; ++i) {   // few: the largest, k times (equal ones go together: a lower bound then)
            uint32_t most = 0;
#pragma unroll
            for (int n = 0; n < T / 32; ++n) most = max(most, own[n]);
            bound = __reduce_max_sync(0xFFFFFFFFu, most);
#pragma unroll
            for (int n = 0; n < T / 32; ++n) own[n] = own[n] == bound ? 0u : own[n];
        }
        for (uint32_t bit = k <= 8 ? 0u : 0x8000u; bit; bit >>= 1) {
            unsigned n = 0;
#pragma unroll
            for (int i = 0; i < T / 32; ++i) n += own[i] >= (bound | bit);
            if (__reduce_add_sync(0xFFFFFFFFu, n) >= (unsigned)k) bound |= bit;
        }
        if (lane == 0) sh.bound = bound;
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    auto offer = [&](float x, int j) {
        if (order_key(x) >> 16 < bound) return;
        const int at = atomicAdd(&sh.count, 1);
        if (at < kTopBuffer) sh.key[at] = top_key(x, j);
    };
    // all vectors of the strips that reach the bound, four a thread on their way
    if (mine >= bound) sh.owner[atomicAdd(&sh.strips, 1)] = tid;
    __syncthreads();
    const int length = (row.vecs + T - 1) / T, items = sh.strips * length;
    for (int at = tid; at < items; at += 4 * T) {
        uint4 raw[4];
        int v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int item = at + u * T;
            v[u] = item < items ? sh.owner[item / length] + item % length * T : row.vecs;
            if (v[u] < row.vecs) raw[u] = row.vectors()[v[u]];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (v[u] >= row.vecs) continue;
            float f[Row<DT>::kVec];
            unpack_vector<DT>(raw[u], f);
#pragma unroll
            for (int i = 0; i < Row<DT>::kVec; ++i) offer(f[i], row.first + row.head + v[u] * Row<DT>::kVec + i);
        }
    }
    if (edge >= 0) offer(row.at(edge), row.first + edge);
    __syncthreads();
    int n = sh.count;
    __syncthreads();
    if (n <= kTopBuffer) {
        top_rank(sh, n, k);
        return;
    }
    // Many elements at the bound (equal logits, say): the row in order, 1024 elements at a time, against the k-th best so
    // far.  Equal logits come in rising index, so a full list rejects them.
    constexpr int kStep = 1024;
    unsigned long long least = 0;
    if (tid == 0) sh.count = 0;
    for (int base = 0; base < row.n; base += kStep) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kStep / T; ++i) {
            const int j = base + tid + i * T;
            if (j >= row.n) continue;
            const unsigned long long key = top_key(row.at(j), row.first + j);
            if (key > least) sh.key[atomicAdd(&sh.count, 1)] = key;
        }
        __syncthreads();
        n = sh.count;
        if (n <= k && base + kStep < row.n) continue;
        top_rank(sh, n, k);
        if (tid < k && tid < n) sh.key[tid] = sh.best[tid];   // (a thread for each: k is at most T)
        if (tid == 0) sh.count = min(n, k);
        if (n >= k) least = sh.best[k - 1];
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------------------------------
struct Logits {
    const void *x;
    int64_t ld, rows;
    int vocab, it;
    float scale, c;   // c = scale * log2 e
    unsigned *d_status;
};
struct TokenOut {
    const void *targets;
    float *logprob, *entropy, *lse, *saved, *top_logprob;
    void *top_index;
    int top_k;
};
struct TeacherList {
    const void *index;
    const float *value;
    int64_t ld_index, ld_value;
    int listed, rest;
};

__device__ __forceinline__ int64_t load_index(const void *p, int it, int64_t i)
{
    return it == FP8_I64 ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

// A row's vectors in batches of four a thread: whole ones, then what is left.  A batch is on its way while the one before is
// worked on.  (Ordinary loads: a gradient may be written over its logits.)
constexpr int kBatch = 4;
template <int DT, int T>
struct Batches {
    const uint4 *src;     // the thread's first vector
    int vecs, whole;      // whole: batches without a gap
    __device__ __forceinline__ explicit Batches(const Row<DT> &row)
        : src(row.vectors() + threadIdx.x), vecs(row.vecs), whole(row.vecs / (kBatch * T))
    {
    }
    // batches in all; the vectors of batch b that some thread has
    __device__ __forceinline__ int count() const { return (vecs + kBatch * T - 1) / (kBatch * T); }
    __device__ __forceinline__ int filled(int b) const { return b < whole ? kBatch : (vecs - b * (kBatch * T) + T - 1) / T; }
    __device__ __forceinline__ void load(int b, uint4 (&raw)[kBatch]) const
    {
        const uint4 *at = src + b * (kBatch * T);
        if (b < whole) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) raw[u] = at[u * T];
        } else if (b == whole) {
            const int left = vecs - b * (kBatch * T) - (int)threadIdx.x;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) raw[u] = u * T < left ? at[u * T] : no_vector<DT>();
        }
    }
    // f(b, vectors) for all batches; `raw`: batch 0, loaded
    template <typename F>
    __device__ __forceinline__ void each(uint4 (&raw)[kBatch], F f) const
    {
        const int n = count();
        uint4 other[kBatch];
        for (int b = 0; b < n; b += 2) {
            load(b + 1, other);
            f(b, raw);
            if (b + 1 >= n) break;
            load(b + 2, raw);
            f(b + 1, other);
        }
    }
};

// One row's elements into sums (relative to a number near the largest), and its largest element.  Bound by the memory as long
// as an element costs few instructions (an SM issues ten of them in the time that an element's two bytes take): two of
// everything an instruction where there is such a one, one exponential, the largest of 32 packed elements looked at once.
// `hide(v, vector)` may take elements out of vector v.
template <int DT, int T, bool ENTROPY, typename Hide>
__device__ __forceinline__ Sums stream_row(const Row<DT> &row, float c, uint4 (&first)[kBatch], float &top, Hide hide)
{
    constexpr int kPairs = kVecPairs<DT>;
    const Pair c2 = pair_of(c);
    Sums a = no_sums();
    Pair s = pair_of(0.0f), t = pair_of(0.0f), less = pair_of(FLT_MAX);
    top = -INFINITY;
    const Batches<DT, T> batches(row);
    batches.each(first, [&](int b, uint4 (&raw)[kBatch]) {
        const int filled = batches.filled(b);
        uint32_t most = no_vector<DT>().x;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u >= filled) continue;
            hide(b * (kBatch * T) + u * T, raw[u]);
            most = max_packed<DT>(most, max_packed<DT>(max_packed<DT>(raw[u].x, raw[u].y), max_packed<DT>(raw[u].z, raw[u].w)));
        }
        const float here = packed_top<DT>(most);
        top = fmaxf(top, here);
        if ((here - a.m) * c > kLead) {
            a.s = sum_of(s);
            a.t = sum_of(t);
            a.relate(here, c);
            s = make_pair(a.s, 0.0f);
            t = make_pair(a.t, 0.0f);
            less = pair_of(-a.m);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u >= filled) continue;
            Pair x[kPairs];
            unpack_pairs<DT>(raw[u], x);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                Pair d = (x[i] + less) * c2;
                float lo, hi;
                split(d, lo, hi);
                if (ENTROPY) {   // (0 * -infinity)
                    lo = max_nan(lo, kFloor);
                    hi = max_nan(hi, kFloor);
                    d = make_pair(lo, hi);
                }
                const Pair e = make_pair(exp2_approx(lo), exp2_approx(hi));
                s = s + e;
                if (ENTROPY) t = fma(e, d, t);
            }
        }
    });
    a.s = sum_of(s);
    a.t = sum_of(t);
    return a;
}

// ---------------------------------------------------------------------------------------------------------------------
// clusters: a row in as many parts as there are blocks
// ---------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(const void *p, unsigned block)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(block));
    return r;
}
// The first elements of block b's part (b = blocks: the row's end): whole 64s.
__device__ __forceinline__ int part_start(int vocab, int blocks, int b)
{
    if (blocks == 1) return b * vocab;
    const int chunk = (vocab / blocks + 64) & ~63;
    return min(vocab, b * chunk);
}
// Sums of all the parts, for the first block, behind a cluster_sync that follows the parts' words.
__device__ __forceinline__ void cluster_note(const Sums &own, float4 &word)
{
    if (threadIdx.x == 0) word = make_float4(own.m, own.s, own.t, 0.0f);
}
__device__ __forceinline__ Sums cluster_join(int blocks, float c, const float4 &word)
{
    Sums all = no_sums();
    float most = -INFINITY;
    for (int b = 0; b < blocks; ++b) {
        Sums o;
        const uint32_t at = cluster_address(&word, b);
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(o.m), "=f"(o.s) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.t) : "r"(at + 8) : "memory");
        most = fmaxf(most, o.m);
        if (o.s != 0.0f) all.join(o, c);
    }
    all.m = most;
    return all;
}

// A row (or a part of one) a block.  4096 x 50257 BF16, 412 MB: 74 us from a graph (5.6 TB/s); an element takes 7.6 instructions
// and one exponential, which is 49 us of the units for those at 1.76 GHz, and rows of sixteen blocks an SM come in 1.7 rounds.
// 512 x 128256 FP32 with 20 top tokens, 263 MB: 60 us.  Tried: 32 threads a row (as quick, slower where an SM has few rows); batches
// of 2, 3 and 6 vectors, 10 and 12 blocks of 128 threads an SM (no better); copies to a ring in shared memory instead of registers
// (8.4 instructions an element, 2 to 5 % slower).
template <int DT, int T>
__global__ void __launch_bounds__(T, 1024 / T) token_logprobs_kernel(const Logits p, const TokenOut o, int blocks)
{
    __shared__ TopShared<T> top;
    __shared__ JoinShared<T> part;
    __shared__ float4 word;
    const int64_t r = blockIdx.x / (unsigned)blocks;
    const int own = (int)(blockIdx.x % (unsigned)blocks), from = part_start(p.vocab, blocks, own);
    const Row<DT> row(p.x, r * p.ld, from, part_start(p.vocab, blocks, own + 1) - from);
    uint4 raw[kBatch];
    Batches<DT, T>(row).load(0, raw);
    // the given token's logit, on its way while the row is read
    int64_t given = -1;
    float given_logit = 0.0f;
    if (o.logprob && own == 0 && threadIdx.x == 0) {
        given = load_index(o.targets, p.it, r);
        if (given >= 0 && given < p.vocab) given_logit = load1<DT>(p.x, r * p.ld + given);
    }
    float strip;   // the thread's largest element
    Sums sums = stream_row<DT, T, true>(row, p.c, raw, strip, [](int, uint4 &) {});
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0) {
        const float x = row.at(edge);
        add_element<true>(sums, x, p.c);
        strip = fmaxf(strip, x);
    }
    sums = block_join<T>(sums, strip, p.c, part);
    if constexpr (T > 64)
        if (o.top_k > 0) find_top<DT, T>(row, strip, o.top_k, top);   // (of a row with a NaN too: what it finds there is not used)
    if (blocks > 1) {
        cluster_note(sums, word);
        cluster_sync();
        if (own == 0) sums = cluster_join(blocks, p.c, word);
    }
    // nothing but -infinity: s = 0;  a NaN or +infinity: s is NaN
    const bool none = sums.s == 0.0f, nan = !(sums.s >= 0.0f);
    const float logsum = none ? -INFINITY : logf(sums.s);
    if (own == 0 && threadIdx.x == 0) {
        const float h = none ? 0.0f : logsum - kLn2 * (sums.t / sums.s);
        if (o.entropy) o.entropy[r] = h;
        if (o.lse) o.lse[r] = none ? -INFINITY : __fmaf_rn(p.scale, sums.m, logsum);
        if (o.saved) reinterpret_cast<float4 *>(o.saved)[r] = make_float4(none ? 0.0f : sums.m, none ? INFINITY : logsum, h, none ? INFINITY : logsum);
        if (o.logprob) {
            float lp = 0.0f;
            if (given >= p.vocab) {
                raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
                lp = NAN;
            } else if (given >= 0) {
                lp = none ? -INFINITY : p.scale * (given_logit - sums.m) - logsum;
            }
            o.logprob[r] = lp;
        }
    }
    if constexpr (T > 64) {
        if (o.top_k > 0 && own == 0) {
            if (blocks > 1) {
                for (int i = threadIdx.x; i < blocks * o.top_k; i += T) {
                    const uint32_t at = cluster_address(&top.best[i % o.top_k], i / o.top_k);
                    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(top.key[i]) : "r"(at) : "memory");
                }
                __syncthreads();
                top_rank(top, blocks * o.top_k, o.top_k);
            }
            for (int i = threadIdx.x; i < o.top_k; i += T) {
                const int64_t at = r * o.top_k + i;
                const unsigned long long key = nan ? 0 : top.best[i];
                const int j = nan ? -1 : (int)~(uint32_t)key;
                o.top_logprob[at] = nan ? NAN : none ? -INFINITY : p.scale * (order_value((uint32_t)(key >> 32)) - sums.m) - logsum;
                if (p.it == FP8_I64) static_cast<int64_t *>(o.top_index)[at] = j;
                else static_cast<int32_t *>(o.top_index)[at] = j;
            }
        }
    }
    if (blocks > 1) cluster_sync();   // (no block leaves while another reads its words)
}

// A row's list: thread i holds entry i.  What of it is worked out in one exchange between the warps: q of the entries that
// count, the sum Q of all q and the rest's q (zeros where no entry counts).
struct ListEntry {
    int j;        // token, or -1
    float v;      // its value
    float q, lnq;
    float mass, rest, total;   // sum of q over the list, q of the rest, both
    // no other token can come: what is left goes to none
    __device__ __forceinline__ void drop_rest()
    {
        total = mass;
        rest = 0.0f;
    }
};
// (and a block's vectors more: a thread without a vector looks at its bits all the same)
__host__ __device__ constexpr int list_words(int vocab) { return (vocab + 7 + 31) / 32 + 64; }
template <int T>
struct ListShared {
    int index[T];
    double sum[T / 32];   // of q, or of exp(v - top)
    float top[T / 32];
    int any[T / 32];      // some entry counts, bit 1: a token came twice
};
// The entry, and a bit for each token that is listed: token j at j + shift, so that a vector's bits lie in one word.  Complete
// for all threads after the next barrier.
template <int T>
__device__ __forceinline__ ListEntry note_list(const Logits &p, const TeacherList &l, int64_t r, ListShared<T> &sh, uint32_t *bits, int shift)
{
    const int tid = threadIdx.x;
    ListEntry e = {-1, -INFINITY, 0.0f, -INFINITY, 0.0f, 0.0f, 0.0f};
    int64_t j = -1;
    if (tid < l.listed) {
        j = load_index(l.index, p.it, r * l.ld_index + tid);
        e.v = l.value[r * l.ld_value + tid];
    }
    for (int i = tid; i < list_words(p.vocab); i += T) bits[i] = 0u;
    if (j >= p.vocab) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
    else if (j >= 0) e.j = (int)j;
    sh.index[tid] = e.j;
    __syncthreads();
    bool again = false;
    if (e.j >= 0) {
        const uint32_t bit = 1u << ((e.j + shift) & 31);
        again = atomicOr(&bits[(e.j + shift) >> 5], bit) & bit;
    }
    const bool some = __any_sync(0xFFFFFFFFu, e.j >= 0), twice = __any_sync(0xFFFFFFFFu, again);
    if ((tid & 31) == 0) sh.any[tid >> 5] = (some ? 1 : 0) | (twice ? 2 : 0);
    return e;
}
// The warp's part of the sums over the list, for `share_list` after the next barrier.
template <int T>
__device__ __forceinline__ void sum_list(const TeacherList &l, ListEntry &e, ListShared<T> &sh)
{
    // (64 bits: 1 - sum of q loses what both have in common)
    double sum;
    float top = 0.0f;
    const float v = e.j >= 0 ? e.v : -INFINITY;
    if (l.rest) {
        sum = e.j >= 0 ? exp((double)v) : 0.0;
    } else {
        top = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        sum = e.j >= 0 && top != -INFINITY ? (double)expf(v - top) : 0.0;
    }
    e.q = (float)sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if ((threadIdx.x & 31) == 0) {
        sh.sum[threadIdx.x >> 5] = sum;
        sh.top[threadIdx.x >> 5] = top;
    }
}
template <int T>
__device__ __forceinline__ void share_list(const TeacherList &l, ListEntry &e, ListShared<T> &sh)
{
    int any = sh.any[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) any |= sh.any[i];
    if (any & 2) {   // a token that is listed twice: its first entry counts, and the sums are taken again
        bool again = false;
        for (int i = 0; i < (int)threadIdx.x; ++i) again = again || sh.index[i] == e.j;
        if (again) e.j = -1;
        __syncthreads();
        sum_list<T>(l, e, sh);
        __syncthreads();
    }
    if (!(any & 1)) return;
    double sum = 0.0;
    if (l.rest) {
#pragma unroll
        for (int i = 0; i < T / 32; ++i) sum += sh.sum[i];
        const double rest = sum >= 1.0 ? 0.0 : 1.0 - sum;   // (NaN stays)
        e.lnq = e.v;
        e.mass = (float)sum;
        e.rest = (float)rest;
        e.total = (float)(sum + rest);
        return;
    }
    float top = sh.top[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) top = max_nan(top, sh.top[i]);
    if (top == -INFINITY) {   // q = 0 for all
        e.q = 0.0f;
        return;
    }
#pragma unroll
    for (int i = 0; i < T / 32; ++i)
        if (sh.top[i] != -INFINITY) sum += sh.sum[i] * (double)expf(sh.top[i] - top);
    const float all = (float)sum;
    e.q = e.j >= 0 ? expf(e.v - top) / all : 0.0f;
    e.lnq = (e.v - top) - logf(all);
    e.mass = e.total = all >= 0.0f ? 1.0f : NAN;
}
template <int DT>
__device__ __forceinline__ int list_shift(const Row<DT> &row) { return -(row.first + row.head) & (Row<DT>::kVec - 1); }
// `j`: place in this part of the row
template <int DT>
__device__ __forceinline__ bool is_listed(const uint32_t *bits, const Row<DT> &row, int j)
{
    const int bit = row.first + j + list_shift<DT>(row);
    return bits[bit >> 5] >> (bit & 31) & 1u;
}
// Elements whose bit is set become -infinity.
template <int DT>
__device__ __forceinline__ void hide_bits(uint32_t hidden, uint4 &raw)
{
    uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    const uint32_t no = no_vector<DT>().x;
#pragma unroll
    for (int i = 0; i < Row<DT>::kVec; ++i) {
        if (!(hidden >> i & 1u)) continue;
        if (DT == FP8_F32) w[i % 4] = no;
        else w[i / 2] = i & 1 ? (w[i / 2] & 0x0000FFFFu) | (no & 0xFFFF0000u) : (w[i / 2] & 0xFFFF0000u) | (no & 0x0000FFFFu);
    }
    raw = make_uint4(w[0], w[1], w[2], w[3]);
}
// The thread's view of the bits: those of its vectors lie at one place in words that are as far apart as the vectors.
template <int DT>
struct ListedVectors {
    const uint32_t *word;
    int place;
    __device__ __forceinline__ ListedVectors(const uint32_t *bits, const Row<DT> &row)
    {
        const int bit = row.first + row.head + list_shift<DT>(row) + (int)threadIdx.x * Row<DT>::kVec;
        word = bits + (bit >> 5);
        place = bit & 31;
    }
    // ahead: vectors from the thread's first one (a multiple of the block's threads)
    __device__ __forceinline__ void hide(int ahead, uint4 &raw) const
    {
        const uint32_t hidden = (word[ahead * Row<DT>::kVec / 32] >> place) & ((1u << Row<DT>::kVec) - 1u);
        if (hidden) hide_bits<DT>(hidden, raw);
    }
};

// 2048 x 32000 BF16 with lists of 64, 131 MB: 32.5 us (4.0 TB/s).  Bound by what a row costs beside its elements (the list, two
// joins: some 4 us of latency, which nothing covers at the start and the end of the one round of rows).
template <int DT, int T>
__global__ void __launch_bounds__(T) distill_kernel(const Logits p, const TeacherList l, float *loss, float *saved, int blocks)
{
    extern __shared__ __align__(16) uint32_t listed_bits[];
    __shared__ ListShared<T> sh;
    __shared__ JoinShared<T> part[2];
    __shared__ float4 word;
    __shared__ float terms[T / 32];
    const int64_t r = blockIdx.x / (unsigned)blocks;
    const int own = (int)(blockIdx.x % (unsigned)blocks), from = part_start(p.vocab, blocks, own);
    const Row<DT> row(p.x, r * p.ld, from, part_start(p.vocab, blocks, own + 1) - from);
    uint4 raw[kBatch];
    Batches<DT, T>(row).load(0, raw);   // (on their way while the list is worked out)
    ListEntry e = note_list<T>(p, l, r, sh, listed_bits, list_shift<DT>(row));
    const float x = e.j >= 0 && own == 0 ? load1<DT>(p.x, r * p.ld + e.j) : -INFINITY;
    __syncthreads();
    // the tokens that are not listed, apart from those that are: neither sum is a difference
    const ListedVectors<DT> listed(listed_bits, row);
    float top;
    Sums sums = stream_row<DT, T, false>(row, p.c, raw, top, [&](int ahead, uint4 &raw) { listed.hide(ahead, raw); });
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0 && !is_listed<DT>(listed_bits, row, edge)) {
        const float y = row.at(edge);
        add_element<false>(sums, y, p.c);
        top = fmaxf(top, y);
    }
    if (own == 0) sum_list<T>(l, e, sh);
    Sums others = block_join<T>(sums, top, p.c, part[0]);   // (a barrier)
    if (blocks > 1) {
        cluster_note(others, word);
        cluster_sync();
        if (own == 0) others = cluster_join(blocks, p.c, word);
    }
    if (own == 0) {
        share_list<T>(l, e, sh);
        const bool counts = e.j >= 0;   // (of a token that came twice one entry is left)
        sums = no_sums();
        if (counts) add_element<false>(sums, x, p.c);
        Sums all = block_join<T>(sums, counts ? x : -INFINITY, p.c, part[1]);
        const float most = fmaxf(all.m, others.m);
        if (others.s != 0.0f) {
            if (all.s == 0.0f) all = no_sums();
            all.join(others, p.c);
        }
        all.m = most;
        const bool none = all.s == 0.0f;
        const float logsum = none ? -INFINITY : logf(all.s);
        // ln of the others' sum relative to the row's largest logit, from the sum relative to their own: it may be far below
        const float logrest = others.s == 0.0f ? -INFINITY : __fmaf_rn(p.scale, others.m - all.m, logf(others.s));
        if (logrest == -INFINITY) e.drop_rest();
        float term = 0.0f;
        if (counts && e.q != 0.0f) term = e.q * (e.lnq - (none || x == -INFINITY ? -INFINITY : p.scale * (x - all.m) - logsum));
        if (threadIdx.x == 0 && e.rest != 0.0f) term += e.rest * (logf(e.rest) - (logrest - logsum));
        if (none && e.total != 0.0f && threadIdx.x == 0) term = INFINITY;
        term = block_sum<T>(term, terms);
        if (threadIdx.x == 0) {
            loss[r] = term;
            if (saved)
                reinterpret_cast<float4 *>(saved)[r] = make_float4(none ? 0.0f : all.m, none ? INFINITY : logsum, 0.0f, none ? INFINITY : logrest);
        }
    }
    if (blocks > 1) cluster_sync();   // (no block leaves while another reads its words)
}

// ---------------------------------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------------------------------
struct GradOut {
    void *dx;
    int64_t ld;
    int same;     // rows of logits and gradient lie alike relative to 16 bytes
    int blocks;   // parts of a row
    AmaxSink sink;
};

// dx_j = 2^d (a + b d) with d = log2 p_j (p relative to the sum that log2sum is of), for all j of a part of a row
// that `hide(ahead, vector)` leaves (the others are written as zeros, and later by their own formula); `skip(j)` is the same
// for elements outside the vectors
template <int DT, int T, bool SLOPE, typename Hide, typename Skip>
__device__ __forceinline__ void write_row(const Row<DT> &row, uint4 (&first)[kBatch], void *out, int64_t at, int same, float m, float c,
                                          float log2sum, float a, float b, uint32_t &key, Hide hide, Skip skip)
{
    constexpr int kPairs = kVecPairs<DT>, kSize = InType<DT>::kBytes;
    auto value = [&](float x) {
        const float d = max_nan(__fmaf_rn(x - m, c, -log2sum), kFloor), e = exp2_approx(d);
        const uint32_t bits = element_bits<DT>(e * (SLOPE ? __fmaf_rn(b, d, a) : a));
        key = max(key, magnitude_key(element_value<DT>(bits)));
        return bits;
    };
    if (!same) {
        for (int j = threadIdx.x; j < row.n; j += T)
            if (!skip(j)) store_bits<DT>(out, at + j, value(row.at(j)));
        return;
    }
    uint32_t acc = 0;
    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(out) + (at + row.head) * kSize) + threadIdx.x;
    const Pair less = pair_of(-m), c2 = pair_of(c), off = pair_of(-log2sum), a2 = pair_of(a), b2 = pair_of(b);
    const Batches<DT, T> batches(row);
    batches.each(first, [&](int n, uint4 (&raw)[kBatch]) {
        const int left = row.vecs - n * (kBatch * T) - (int)threadIdx.x;
        uint4 *to = dst + n * (kBatch * T);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (u * T >= left) continue;
            hide(n * (kBatch * T) + u * T, raw[u]);
            Pair x[kPairs];
            unpack_pairs<DT>(raw[u], x);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                Pair d = fma(x[i] + less, c2, off);
                float lo, hi;
                split(d, lo, hi);
                if (SLOPE) {   // (0 * -infinity)
                    lo = max_nan(lo, kFloor);
                    hi = max_nan(hi, kFloor);
                    d = make_pair(lo, hi);
                }
                const Pair e = make_pair(exp2_approx(lo), exp2_approx(hi));
                x[i] = e * (SLOPE ? fma(b2, d, a2) : a2);
            }
            const uint4 y = pack_pairs<DT>(x);
            acc = fold_vector<DT>(acc, y);
            to[u * T] = y;
        }
    });
    key = max(key, folded_key<DT>(acc));
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0 && !skip(edge)) store_bits<DT>(out, at + edge, value(row.at(edge)));
}

template <int DT, int T>
__device__ __forceinline__ void write_zeros(void *out, int64_t at, int n)
{
    const Row<DT> row(out, at, 0, n);
    uint4 *dst = const_cast<uint4 *>(row.vectors());
    for (int v = threadIdx.x; v < row.vecs; v += T) dst[v] = make_uint4(0u, 0u, 0u, 0u);
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0) store_bits<DT>(out, at + edge, 0u);
}

// 4096 x 32000 BF16, 524 MB read and written: 85 us (6.2 TB/s), bound by the memory.
template <int DT, int T>
__global__ void __launch_bounds__(T) token_logprobs_bwd_kernel(const Logits p, const void *targets, const float *saved,
                                                                          const float *g_lp, int64_t g_lp_stride, const float *g_h,
                                                                          int64_t g_h_stride, const GradOut o)
{
    const int64_t r = blockIdx.x / (unsigned)o.blocks;
    const int part = (int)(blockIdx.x % (unsigned)o.blocks), from = part_start(p.vocab, o.blocks, part);
    const int count = part_start(p.vocab, o.blocks, part + 1) - from;
    const int64_t at = r * o.ld + from;
    const float4 keep = reinterpret_cast<const float4 *>(saved)[r];
    int64_t t = g_lp && targets ? load_index(targets, p.it, r) : -1;
    if (t >= p.vocab) {
        if (threadIdx.x == 0) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
        t = -1;
    }
    const float g = t >= 0 ? g_lp[r * g_lp_stride] : 0.0f, gh = g_h ? g_h[r * g_h_stride] : 0.0f;
    uint32_t key = 0;
    if ((g == 0.0f && gh == 0.0f) || keep.y == INFINITY) {
        write_zeros<DT, T>(o.dx, at, count);
    } else {
        const Row<DT> row(p.x, r * p.ld, from, count);
        uint4 raw[kBatch];
        Batches<DT, T>(row).load(0, raw);
        const int given = t >= from && t < from + count ? (int)t - from : -1;   // this part's
        uint32_t own = 0;
        if (given >= 0 && threadIdx.x == 0) {
            // 1 - p of a token that is nearly certain: expm1 keeps its digits
            const float lp = max_nan(p.scale * (row.at(given) - keep.x) - keep.y, -1e30f), prob = expf(lp);
            own = element_bits<DT>(p.scale * (-g * expm1f(lp) - gh * prob * (lp + keep.z)));
        }
        __syncthreads();   // (the gradient may overwrite the logits)
        const int given_vec = given >= row.head ? (given - row.head) / Row<DT>::kVec - (int)threadIdx.x : -1;
        const int given_bit = (given - row.head) % Row<DT>::kVec;
        write_row<DT, T, true>(row, raw, o.dx, at, o.same, keep.x, p.c, keep.y * kLog2e, p.scale * (-g - gh * keep.z), -p.scale * gh * kLn2, key,
                            [&](int ahead, uint4 &raw) {
                                if (ahead == given_vec) hide_bits<DT>(1u << given_bit, raw);
                            },
                            [&](int j) { return j == given; });
        __syncthreads();
        if (given >= 0 && threadIdx.x == 0) {
            store_bits<DT>(o.dx, at + given, own);
            key = max(key, magnitude_key(element_value<DT>(own)));
        }
    }
    sink_amax(key, o.sink);
}

// Unlisted tokens far below the row's largest logit (a finite mask on all of them): of the difference of two such distances no digit
// may be left, so their own largest and sum are taken again, by all parts of the row, before one of them writes: dx_j = a s_j.
// (Element by element and a call: few rows come here, and the others' code stays as it is.)
template <int DT, int T>
__device__ __noinline__ uint32_t write_far_rest(const Row<DT> row, const uint32_t *bits, void *out, int64_t at, int blocks, float c, float a,
                                                JoinShared<T> &joint, float4 &word)
{
    uint32_t key = 0;
    Sums others = no_sums();
    float top = -INFINITY;
    for (int j = threadIdx.x; j < row.n; j += T) {
        if (is_listed<DT>(bits, row, j)) continue;
        const float x = row.at(j);
        add_element<false>(others, x, c);
        top = fmaxf(top, x);
    }
    others = block_join<T>(others, top, c, joint);
    if (blocks > 1) {
        cluster_note(others, word);
        cluster_sync();
        others = cluster_join(blocks, c, word);
    }
    const float log2sum = logf(others.s) * kLog2e;
    for (int j = threadIdx.x; j < row.n; j += T) {
        if (is_listed<DT>(bits, row, j)) continue;
        const uint32_t v = element_bits<DT>(a * exp2_approx(__fmaf_rn(row.at(j) - others.m, c, -log2sum)));
        key = max(key, magnitude_key(element_value<DT>(v)));
        store_bits<DT>(out, at + j, v);
    }
    if (blocks > 1) cluster_sync();   // (no block leaves while another reads its word)
    return key;
}

// 2048 x 50257 FP16 with lists of 32, 412 MB read and written: 73 us (5.6 TB/s), bound by the memory and the list's latency.
template <int DT, int T>
__global__ void __launch_bounds__(T) distill_bwd_kernel(const Logits p, const TeacherList l, const float *saved,
                                                                   const float *g_loss, int64_t g_stride, const GradOut o)
{
    extern __shared__ __align__(16) uint32_t listed_bits[];
    __shared__ ListShared<T> sh;
    __shared__ JoinShared<T> joint;
    __shared__ float4 word;
    const int64_t r = blockIdx.x / (unsigned)o.blocks;
    const int part = (int)(blockIdx.x % (unsigned)o.blocks), from = part_start(p.vocab, o.blocks, part);
    const int count = part_start(p.vocab, o.blocks, part + 1) - from;
    const int64_t at = r * o.ld + from;
    const float4 keep = reinterpret_cast<const float4 *>(saved)[r];
    const float g = g_loss[r * g_stride] * p.scale;
    uint32_t key = 0;
    if (g == 0.0f || keep.y == INFINITY) {
        write_zeros<DT, T>(o.dx, at, count);
    } else {
        const Row<DT> row(p.x, r * p.ld, from, count);
        uint4 raw[kBatch];
        Batches<DT, T>(row).load(0, raw);   // (on their way while the list is worked out)
        ListEntry e = note_list<T>(p, l, r, sh, listed_bits, list_shift<DT>(row));
        const float x = e.j >= from && e.j < from + count ? row.at(e.j - from) : 0.0f;
        sum_list<T>(l, e, sh);
        __syncthreads();   // (also: the gradient may overwrite the logits)
        share_list<T>(l, e, sh);
        if (keep.w == -INFINITY) e.drop_rest();
        if (e.total == 0.0f) {   // no entry counts: the loss is 0, whatever the logits are
            write_zeros<DT, T>(o.dx, at, count);
            sink_amax(key, o.sink);
            return;
        }
        const int own_j = e.j >= from && e.j < from + count ? e.j - from : -1;
        uint32_t own = 0;
        if (own_j >= 0) {
            const float prob = expf(p.scale * (x - keep.x) - keep.y);
            own = element_bits<DT>(g * __fmaf_rn(e.total, prob, -e.q));
        }
        // the others: p_j Q, or with s_j = p_j / p_r, s_j (Q p_r - q_r): s_j is one of a sum of 1 however small p_r is
        const float a = e.rest == 0.0f ? e.total : __fmaf_rn(e.total, expf(keep.w - keep.y), -e.rest);
        if (e.rest != 0.0f && keep.w < kFarRest) {
            key = write_far_rest<DT, T>(row, listed_bits, o.dx, at, o.blocks, p.c, g * a, joint, word);
        } else {
            const float logsum = e.rest == 0.0f ? keep.y : keep.w;
            const ListedVectors<DT> listed(listed_bits, row);
            write_row<DT, T, false>(row, raw, o.dx, at, o.same, keep.x, p.c, logsum * kLog2e, g * a, 0.0f, key,
                                 [&](int ahead, uint4 &raw) { listed.hide(ahead, raw); },
                                 [&](int j) { return is_listed<DT>(listed_bits, row, j); });
        }
        __syncthreads();
        if (own_j >= 0) {
            store_bits<DT>(o.dx, at + own_j, own);
            key = max(key, magnitude_key(element_value<DT>(own)));
        }
    }
    sink_amax(key, o.sink);
}

// ---------------------------------------------------------------------------------------------------------------------
// calls
// ---------------------------------------------------------------------------------------------------------------------
static fp8_status_t check_logits(const fp8_ctx *ctx, const void *logits, int dt, int64_t ld, int64_t rows, int64_t vocab, float scale, int it)
{
    if (!ctx || !logits) return FP8_ERR_NULL;
    if (dt < 0 || dt > 2 || it < 0 || it > 1) return FP8_ERR_DTYPE;
    if (rows <= 0 || rows > 0x7FFFFFFF || vocab <= 0 || vocab > 1 << 30 || ld < vocab) return FP8_ERR_SHAPE;
    if (!(scale > 0.0f && scale * kLog2e <= FLT_MAX)) return FP8_ERR_SHAPE;
    return element_aligned(logits, dt) ? FP8_OK : FP8_ERR_ALIGN;
}
static bool index_aligned(const void *p, int it) { return (reinterpret_cast<uintptr_t>(p) & (it == FP8_I64 ? 7u : 3u)) == 0; }
static bool float_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static bool saved_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static fp8_status_t check_list(const void *index, int it, int64_t ld_index, const float *value, int64_t ld_value, int listed, int mode)
{
    if (!index || !value) return FP8_ERR_NULL;
    if (mode < 0 || mode > 1) return FP8_ERR_DTYPE;
    if (listed <= 0 || ld_index < listed || ld_value < listed) return FP8_ERR_SHAPE;
    if (listed > FP8_LOSS_LISTED_MAX) return FP8_ERR_UNSUPPORTED;
    return index_aligned(index, it) && float_aligned(value) ? FP8_OK : FP8_ERR_ALIGN;
}

static Logits make_logits(const fp8_ctx *ctx, const void *x, int64_t ld, int64_t rows, int64_t vocab, float scale, int it)
{
    return Logits{x, ld, rows, (int)vocab, it, scale, scale * kLog2e, ctx->d_status};
}

static GradOut make_grad(fp8_ctx *ctx, const void *x, int64_t ld, int dt, void *dx, int64_t ld_d, float *d_amax, int blocks)
{
    const int64_t size = dt == FP8_F32 ? 4 : 2;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(x) & 15u) - (int64_t)(reinterpret_cast<uintptr_t>(dx) & 15u);
    const int same = apart == 0 && (ld - ld_d) * size % 16 == 0;
    return GradOut{dx, ld_d, same, blocks, {d_amax ? take_slot(ctx) : nullptr, d_amax, nullptr, ctx->d_status, FP8_E5, 0, 0}};
}

// In how many parts rows are read: as many blocks as give every SM two of them, of 2048 elements at least.  Parts of a
// forward pass meet once more at the end, which costs more than a shorter last round of blocks gains (4096 rows of 50257: 74, 88
// and 121 us in one, two and four parts; 512 of 128256 with top tokens: 60 and 65); those of a gradient do not, and are cut as long as
// they have 16000 elements (2048 of 50257: 78, 72, 73 us; 4096 of 32000: 87, 84, 90).
static int row_blocks(const fp8_ctx *ctx, int64_t rows, int64_t vocab, bool join)
{
    int blocks = 1;
    while (blocks < 8 && ((rows * blocks < (int64_t)ctx->sm_count * 2 && vocab / (2 * blocks) >= 2048) || (!join && vocab / (2 * blocks) >= 16000)))
        blocks *= 2;
    return blocks;
}

// Threads of a row's block: `least` of them at least, and as many as let an SM's shared memory (`shared` bytes a block) hold 1024
// threads.  Sixteen rows an SM by 64 threads come in half as many rounds as eight by 128, each of which has its latencies at both
// ends (forward, 8192 rows of 50257: 134 and 144 us; 4096: 74 and 78; 2048 of 32000 with lists of 64: 32.5 and 35).  By shared
// memory: 2048 rows of 262144 with lists take 178 us by 256 threads and 220 by 128, their gradient 325 and 406.
static int row_threads(int least, unsigned shared)
{
    int threads = least <= 64 ? 64 : least <= 128 ? 128 : 256;
    while (threads < 256 && 1024u / threads * (shared + 2048u) > 227u << 10) threads *= 2;
    return threads;
}
// Where there are no eight rows an SM, 256 (forward, 512 rows of 128256 with top tokens: 60 us; by 128 threads 103).
static int few_row_threads(const fp8_ctx *ctx, int64_t rows, int blocks) { return rows * blocks < (int64_t)ctx->sm_count * 8 ? 256 : 1; }

// `cluster`: the blocks of a row are one.
template <typename... KArgs, typename... Args>
static fp8_status_t launch_rows(void (*kernel)(KArgs...), int threads, int64_t rows, int blocks, bool cluster, unsigned smem, void *stream, Args... args)
{
    if (rows * blocks > 0x7FFFFFFF) return FP8_ERR_SHAPE;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * blocks));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr;
    cfg.numAttrs = cluster && blocks > 1 ? 1 : 0;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...) == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

template <int DT, int T>
static cudaError_t allow_lists()
{
    const int bytes = list_words(FP8_LOSS_VOCAB_MAX) * 4;
    const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    const cudaError_t e = cudaFuncSetAttribute(distill_kernel<DT, T>, attr, bytes);
    if constexpr (T > 64) return e == cudaSuccess ? cudaFuncSetAttribute(distill_bwd_kernel<DT, T>, attr, bytes) : e;
    return e;
}
cudaError_t configure_loss_kernels()
{
    cudaError_t e = allow_lists<FP8_BF16, 64>();
    if (e == cudaSuccess) e = allow_lists<FP8_F16, 64>();
    if (e == cudaSuccess) e = allow_lists<FP8_F32, 64>();
    if (e == cudaSuccess) e = allow_lists<FP8_BF16, 128>();
    if (e == cudaSuccess) e = allow_lists<FP8_BF16, 256>();
    if (e == cudaSuccess) e = allow_lists<FP8_F16, 128>();
    if (e == cudaSuccess) e = allow_lists<FP8_F16, 256>();
    if (e == cudaSuccess) e = allow_lists<FP8_F32, 128>();
    return e == cudaSuccess ? allow_lists<FP8_F32, 256>() : e;
}

}  // namespace fp8lin

#define FP8LIN_LAUNCH_OF(DT, T, KERNEL, ...) launch_rows(KERNEL<DT, T>, T, __VA_ARGS__)
#define FP8LIN_LAUNCH_BY_TYPE(T, KERNEL, ...)                                                          \
    (dt == FP8_BF16  ? FP8LIN_LAUNCH_OF(FP8_BF16, T, KERNEL, __VA_ARGS__)                              \
     : dt == FP8_F16 ? FP8LIN_LAUNCH_OF(FP8_F16, T, KERNEL, __VA_ARGS__)                               \
                     : FP8LIN_LAUNCH_OF(FP8_F32, T, KERNEL, __VA_ARGS__))
#define FP8LIN_LAUNCH_BY_SIZE(THREADS, KERNEL, ...)               \
    ((THREADS) == 64    ? FP8LIN_LAUNCH_BY_TYPE(64, KERNEL, __VA_ARGS__)  \
     : (THREADS) == 128 ? FP8LIN_LAUNCH_BY_TYPE(128, KERNEL, __VA_ARGS__) \
                        : FP8LIN_LAUNCH_BY_TYPE(256, KERNEL, __VA_ARGS__))

extern "C" {

fp8_status_t fp8_token_logprobs(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows, int64_t vocab, float scale,
                                const void *targets, fp8_itype_t it, float *logprob, float *entropy, float *lse, float *saved,
                                int32_t top_k, float *top_logprob, void *top_index, void *stream)
{
    using namespace fp8lin;
    const fp8_status_t s = check_logits(ctx, logits, (int)dt, ld, rows, vocab, scale, (int)it);
    if (s != FP8_OK) return s;
    if (!logprob && !entropy && !lse && !saved && top_k == 0) return FP8_ERR_NULL;
    if (logprob && !targets) return FP8_ERR_NULL;
    if (top_k < 0 || top_k > vocab) return FP8_ERR_SHAPE;
    if (top_k > FP8_LOSS_TOP_MAX) return FP8_ERR_UNSUPPORTED;
    if (top_k > 0 && (!top_logprob || !top_index)) return FP8_ERR_NULL;
    if (!index_aligned(targets, (int)it) || !float_aligned(logprob) || !float_aligned(entropy) || !float_aligned(lse) || !saved_aligned(saved) ||
        !float_aligned(top_logprob) || !index_aligned(top_index, (int)it))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const TokenOut o = {targets, logprob, entropy, lse, saved, top_logprob, top_index, top_k};
    const int blocks = row_blocks(ctx, rows, vocab, true);
    // (top tokens: 64 threads have no place for them, and twice as many strips keep the candidates of a long list few)
    const int threads = row_threads(std::max(few_row_threads(ctx, rows, blocks), top_k == 0 ? 64 : top_k <= 32 ? 128 : 256), 0u);
    return FP8LIN_LAUNCH_BY_SIZE(threads, token_logprobs_kernel, rows, blocks, true, 0u, stream, p, o, blocks);
}

fp8_status_t fp8_token_logprobs_bwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows, int64_t vocab, float scale,
                                    const void *targets, fp8_itype_t it, const float *saved, const float *g_logprob,
                                    int64_t g_logprob_stride, const float *g_entropy, int64_t g_entropy_stride, void *dlogits,
                                    int64_t ld_d, float *d_amax, void *stream)
{
    using namespace fp8lin;
    const fp8_status_t s = check_logits(ctx, logits, (int)dt, ld, rows, vocab, scale, (int)it);
    if (s != FP8_OK) return s;
    if (!saved || !dlogits || (!g_logprob && !g_entropy) || (g_logprob && !targets)) return FP8_ERR_NULL;
    if (ld_d < vocab || g_logprob_stride < 0 || g_entropy_stride < 0) return FP8_ERR_SHAPE;
    if (dlogits == logits && ld_d != ld && rows > 1) return FP8_ERR_SHAPE;
    if (!index_aligned(targets, (int)it) || !saved_aligned(saved) || !float_aligned(g_logprob) || !float_aligned(g_entropy) ||
        !element_aligned(dlogits, (int)dt) || !float_aligned(d_amax))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const int blocks = row_blocks(ctx, rows, vocab, false);
    const GradOut o = make_grad(ctx, logits, ld, (int)dt, dlogits, ld_d, d_amax, blocks);
    return FP8LIN_LAUNCH_BY_TYPE(128, token_logprobs_bwd_kernel, rows, blocks, false, 0u, stream, p, targets, saved, g_logprob, g_logprob_stride,
                                 g_entropy, g_entropy_stride, o);
}

fp8_status_t fp8_distill_fwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows, int64_t vocab, float scale,
                             const void *index, fp8_itype_t it, int64_t ld_index, const float *value, int64_t ld_value, int32_t listed,
                             fp8_distill_mode_t mode, float *loss, float *saved, void *stream)
{
    using namespace fp8lin;
    fp8_status_t s = check_logits(ctx, logits, (int)dt, ld, rows, vocab, scale, (int)it);
    if (s == FP8_OK) s = check_list(index, (int)it, ld_index, value, ld_value, listed, (int)mode);
    if (s != FP8_OK) return s;
    if (!loss) return FP8_ERR_NULL;
    if (vocab > FP8_LOSS_VOCAB_MAX) return FP8_ERR_UNSUPPORTED;
    if (!float_aligned(loss) || !saved_aligned(saved)) return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const TeacherList l = {index, value, ld_index, ld_value, listed, mode == FP8_DISTILL_REST};
    const int blocks = row_blocks(ctx, rows, vocab, true);
    const unsigned shared = list_words((int)vocab) * 4u;
    const int threads = row_threads(std::max(few_row_threads(ctx, rows, blocks), (int)listed), shared);
    return FP8LIN_LAUNCH_BY_SIZE(threads, distill_kernel, rows, blocks, true, shared, stream, p, l, loss, saved, blocks);
}

fp8_status_t fp8_distill_bwd(fp8_ctx *ctx, const void *logits, fp8_dtype_t dt, int64_t ld, int64_t rows, int64_t vocab, float scale,
                             const void *index, fp8_itype_t it, int64_t ld_index, const float *value, int64_t ld_value, int32_t listed,
                             fp8_distill_mode_t mode, const float *saved, const float *g_loss, int64_t g_loss_stride, void *dlogits,
                             int64_t ld_d, float *d_amax, void *stream)
{
    using namespace fp8lin;
    fp8_status_t s = check_logits(ctx, logits, (int)dt, ld, rows, vocab, scale, (int)it);
    if (s == FP8_OK) s = check_list(index, (int)it, ld_index, value, ld_value, listed, (int)mode);
    if (s != FP8_OK) return s;
    if (!saved || !g_loss || !dlogits) return FP8_ERR_NULL;
    if (ld_d < vocab || g_loss_stride < 0) return FP8_ERR_SHAPE;
    if (dlogits == logits && ld_d != ld && rows > 1) return FP8_ERR_SHAPE;
    if (vocab > FP8_LOSS_VOCAB_MAX) return FP8_ERR_UNSUPPORTED;
    if (!saved_aligned(saved) || !float_aligned(g_loss) || !element_aligned(dlogits, (int)dt) || !float_aligned(d_amax)) return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const TeacherList l = {index, value, ld_index, ld_value, listed, mode == FP8_DISTILL_REST};
    const int blocks = row_blocks(ctx, rows, vocab, false);
    const GradOut o = make_grad(ctx, logits, ld, (int)dt, dlogits, ld_d, d_amax, blocks);
    const unsigned shared = list_words((int)vocab) * 4u;
    // (64 threads: 76 us for 2048 rows of 50257 FP16, by 128 they take 72)
    const bool cluster = l.rest;   // (the parts of a row may have to meet)
    return row_threads(std::max(128, (int)listed), shared) == 128
               ? FP8LIN_LAUNCH_BY_TYPE(128, distill_bwd_kernel, rows, blocks, cluster, shared, stream, p, l, saved, g_loss, g_loss_stride, o)
               : FP8LIN_LAUNCH_BY_TYPE(256, distill_bwd_kernel, rows, blocks, cluster, shared, stream, p, l, saved, g_loss, g_loss_stride, o);
}

}  // extern "C"
