// Log probabilities of given tokens with entropy and top tokens, and the divergence from a teacher's listed tokens, each
// with the gradient of the logits.
#include "fp8_loss.h"
#include "kv_common.cuh"
#include "row_common.cuh"

namespace fp8lin {

constexpr int kLossThreads = 256, kLossWarps = kLossThreads / 32;
constexpr int kTopBuffer = 2048;     // candidates for the top tokens of a row
constexpr float kFloor = -200.0f;    // exponents (base 2) below it are zeros: 2^-200 is none of an FP32 sum
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
// a row as head elements up to the first 16-byte boundary, whole vectors, tail elements
// ---------------------------------------------------------------------------------------------------------------------
template <int DT>
struct Row {
    static constexpr int kVec = DT == FP8_F32 ? 4 : 8;
    const uint8_t *base;
    int n, head, vecs, tail;   // tail: the first element behind the vectors
    __device__ __forceinline__ Row(const void *logits, int64_t at, int count)
    {
        constexpr int kSize = InType<DT>::kBytes;
        base = static_cast<const uint8_t *>(logits) + at * kSize;
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

// Running sums over exp(scale (x - m)): with d = c (x - m), c = scale * log2 e:  s = sum 2^d,  t = sum 2^d d.
struct Sums {
    float m, s, t;
    // the sums relative to a larger maximum
    __device__ __forceinline__ void raise(float to, float c)
    {
        const float d = fmaxf((fmaxf(m, -FLT_MAX) - fmaxf(to, -FLT_MAX)) * c, kFloor), f = exp2_approx(d);
        t = f * __fmaf_rn(d, s, t);
        s *= f;
        m = to;
    }
    template <bool ENTROPY>
    __device__ __forceinline__ void add(float x, float c)
    {
        const float d = max_nan((x - fmaxf(m, -FLT_MAX)) * c, kFloor), e = exp2_approx(d);
        s += e;
        if (ENTROPY) t = __fmaf_rn(e, d, t);
    }
    __device__ __forceinline__ void join(const Sums &o, float c)
    {
        Sums b = o;
        const float to = fmaxf(m, b.m);
        raise(to, c);
        b.raise(to, c);
        s += b.s;
        t += b.t;
    }
};

// Sums over the block, to all threads, always in the same order.
__device__ __forceinline__ Sums block_join(Sums a, float c, Sums *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Sums b = {__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o), __shfl_xor_sync(0xFFFFFFFFu, a.t, o)};
        a.join(b, c);
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int i = 1; i < kLossWarps; ++i) a.join(part[i], c);
    return a;
}

// ---------------------------------------------------------------------------------------------------------------------
// top tokens
// ---------------------------------------------------------------------------------------------------------------------
// Orders like the numbers (-0 like 0); 0 is below every number's key.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x == 0.0f ? 0.0f : x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// larger logit first, then lower index
__device__ __forceinline__ unsigned long long top_key(float x, int j) { return ((unsigned long long)order_key(x) << 32) | (uint32_t)~j; }

struct TopShared {
    unsigned long long key[kTopBuffer];
    uint32_t strip[kLossThreads];
    int count;
    uint32_t bound;
};

// The k largest of sh.key[0 .. n), in order, to the front of the buffer.  Keys differ, so a key's place is the number
// of larger ones.
__device__ __forceinline__ void top_rank(TopShared &sh, int n, int k)
{
    constexpr int kMine = kTopBuffer / kLossThreads;
    unsigned long long mine[kMine];
    int place[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x + i * kLossThreads;
        place[i] = k;
        if (i * kLossThreads >= n) continue;
        mine[i] = at < n ? sh.key[at] : ~0ull;
        int larger = 0;
        for (int o = 0; o < n; ++o) larger += sh.key[o] > mine[i];
        place[i] = at < n ? larger : k;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (place[i] < k) sh.key[place[i]] = mine[i];
    __syncthreads();
}

// The row's top k keys into sh.key[0 .. k).  m: the thread's own largest element (its strip: the vectors v = thread mod
// block size, and its edge element).  A bound that k strips reach is reached by k elements; only those strips are read again.
template <int DT>
__device__ __forceinline__ void find_top(const Row<DT> &row, float m, int k, TopShared &sh)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int edge = row.edge(tid);
    // sixteen bits of the key are enough of a bound
    const uint32_t mine = tid < row.vecs || edge >= 0 ? order_key(m) >> 16 : 0u;
    sh.strip[tid] = mine;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (warp == 0) {
        uint32_t own[kLossWarps], bound = 0;
#pragma unroll
        for (int i = 0; i < kLossWarps; ++i) own[i] = sh.strip[lane + 32 * i];
        for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
            unsigned n = 0;
#pragma unroll
            for (int i = 0; i < kLossWarps; ++i) n += own[i] >= (bound | bit);
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
    unsigned flagged = __ballot_sync(0xFFFFFFFFu, mine >= bound);
    while (flagged) {
        const int owner = (warp << 5) + __ffs(flagged) - 1;
        flagged &= flagged - 1;
        for (int v = owner + lane * kLossThreads; v < row.vecs; v += 32 * kLossThreads) {
            float f[Row<DT>::kVec];
            unpack_vector<DT>(__ldg(row.vectors() + v), f);
#pragma unroll
            for (int i = 0; i < Row<DT>::kVec; ++i) offer(f[i], row.head + v * Row<DT>::kVec + i);
        }
    }
    if (edge >= 0) offer(row.at(edge), edge);
    __syncthreads();
    int n = sh.count;
    __syncthreads();
    if (n <= kTopBuffer) {
        top_rank(sh, n, k);
        return;
    }
    // Many elements at the bound (equal logits, say): the row in order, 1024 elements at a time, against the k-th best so
    // far.  Equal logits come in rising index, so a full list rejects them.
    unsigned long long least = 0;
    if (tid == 0) sh.count = 0;
    for (int base = 0; base < row.n; base += 4 * kLossThreads) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = base + tid + i * kLossThreads;
            if (j >= row.n) continue;
            const unsigned long long key = top_key(row.at(j), j);
            if (key > least) sh.key[atomicAdd(&sh.count, 1)] = key;
        }
        __syncthreads();
        n = sh.count;
        if (n <= k && base + 4 * kLossThreads < row.n) continue;
        __syncthreads();
        top_rank(sh, n, k);
        if (tid == 0) sh.count = min(n, k);
        if (n >= k) least = sh.key[k - 1];
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

// One row's elements through `sums`; `hide(v, vector)` may take elements out of a vector first.
template <int DT, bool ENTROPY, typename Hide>
__device__ __forceinline__ void stream_row(const Row<DT> &row, float c, Sums &sums, Hide hide)
{
    constexpr int kVec = Row<DT>::kVec, kUnroll = 4;
    for (int v0 = threadIdx.x; v0 < row.vecs; v0 += kUnroll * kLossThreads) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int v = v0 + u * kLossThreads;
            raw[u] = v < row.vecs ? __ldg(row.vectors() + v) : no_vector<DT>();
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float f[kVec];
            hide(v0 + u * kLossThreads, raw[u]);
            unpack_vector<DT>(raw[u], f);
            float top = f[0];
#pragma unroll
            for (int i = 1; i < kVec; ++i) top = fmaxf(top, f[i]);
            if (top > sums.m) sums.raise(top, c);
#pragma unroll
            for (int i = 0; i < kVec; ++i) sums.add<ENTROPY>(f[i], c);
        }
    }
}

template <int DT>
__global__ void __launch_bounds__(kLossThreads) token_logprobs_kernel(const Logits p, const TokenOut o)
{
    __shared__ TopShared top;
    __shared__ Sums part[kLossWarps];
    const int64_t r = blockIdx.x;
    const Row<DT> row(p.x, r * p.ld, p.vocab);
    Sums sums = {-INFINITY, 0.0f, 0.0f};
    stream_row<DT, true>(row, p.c, sums, [](int, uint4 &) {});
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0) {
        const float x = row.at(edge);
        if (x > sums.m) sums.raise(x, p.c);
        sums.add<true>(x, p.c);
    }
    const float strip = sums.m;
    sums = block_join(sums, p.c, part);
    // nothing but -infinity: s = 0;  a NaN or +infinity: s is NaN
    const bool none = sums.s == 0.0f, nan = !(sums.s >= 0.0f);
    const float logsum = none ? -INFINITY : logf(sums.s);
    if (threadIdx.x == 0) {
        const float h = none ? 0.0f : logsum - kLn2 * (sums.t / sums.s);
        if (o.entropy) o.entropy[r] = h;
        if (o.lse) o.lse[r] = none ? -INFINITY : __fmaf_rn(p.scale, sums.m, logsum);
        if (o.saved) reinterpret_cast<float4 *>(o.saved)[r] = make_float4(none ? 0.0f : sums.m, none ? INFINITY : logsum, h, none ? INFINITY : logsum);
        if (o.logprob) {
            const int64_t t = load_index(o.targets, p.it, r);
            float lp = 0.0f;
            if (t >= p.vocab) {
                raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
                lp = NAN;
            } else if (t >= 0) {
                lp = none ? -INFINITY : p.scale * (row.at((int)t) - sums.m) - logsum;
            }
            o.logprob[r] = lp;
        }
    }
    if (o.top_k == 0) return;
    if (!nan) find_top<DT>(row, strip, o.top_k, top);
    for (int i = threadIdx.x; i < o.top_k; i += kLossThreads) {
        const int64_t at = r * o.top_k + i;
        const unsigned long long key = nan ? 0 : top.key[i];
        const int j = nan ? -1 : (int)~(uint32_t)key;
        o.top_logprob[at] = nan ? NAN : none ? -INFINITY : p.scale * (order_value((uint32_t)(key >> 32)) - sums.m) - logsum;
        if (p.it == FP8_I64) static_cast<int64_t *>(o.top_index)[at] = j;
        else static_cast<int32_t *>(o.top_index)[at] = j;
    }
}

// A row's list: thread i holds entry i.  Entries that count, their q and ln q, the sum Q of all q and the rest's q
// (zeros where no entry counts).
struct ListEntry {
    int j;        // token, or -1
    float q, lnq;
    float mass, rest, total;   // sum of q over the list, q of the rest, both
    // no other token can come: what is left goes to none
    __device__ __forceinline__ void drop_rest()
    {
        total = mass;
        rest = 0.0f;
    }
};
struct ListShared {
    int index[kLossThreads];
    float part[kLossWarps];
    double sum[kLossWarps];
};
__device__ __forceinline__ ListEntry load_list(const Logits &p, const TeacherList &l, int64_t r, ListShared &sh)
{
    const int tid = threadIdx.x;
    ListEntry e = {-1, 0.0f, -INFINITY, 0.0f, 0.0f, 0.0f};
    float v = -INFINITY;
    if (tid < l.listed) {
        const int64_t j = load_index(l.index, p.it, r * l.ld_index + tid);
        v = l.value[r * l.ld_value + tid];
        if (j >= p.vocab) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
        else if (j >= 0) e.j = (int)j;
    }
    sh.index[tid] = e.j;
    __syncthreads();
    if (tid < l.listed && e.j >= 0) {
        bool again = false;
        for (int i = 0; i < tid; ++i) again = again || sh.index[i] == e.j;
        if (again) e.j = -1;
    }
    if (e.j < 0) v = -INFINITY;
    if (!__syncthreads_or(e.j >= 0)) return e;   // nothing listed
    if (l.rest) {
        // 1 - sum of q loses what both have in common: in 64 bits
        double q = e.j >= 0 ? exp((double)v) : 0.0;
        e.q = (float)q;
        e.lnq = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
        if ((tid & 31) == 0) sh.sum[tid >> 5] = q;
        __syncthreads();
        q = 0.0;
        for (int i = 0; i < kLossWarps; ++i) q += sh.sum[i];
        const double rest = q >= 1.0 ? 0.0 : 1.0 - q;   // (NaN stays)
        e.mass = (float)q;
        e.rest = (float)rest;
        e.total = (float)(q + rest);
    } else {
        float top = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if ((tid & 31) == 0) sh.part[tid >> 5] = top;
        __syncthreads();
        top = sh.part[0];
        for (int i = 1; i < kLossWarps; ++i) top = max_nan(top, sh.part[i]);
        __syncthreads();
        const bool none = top == -INFINITY;
        float q = none ? 0.0f : expf(v - top);
        const float sum = block_sum<kLossThreads>(q, sh.part);
        e.q = none ? 0.0f : q / sum;
        e.lnq = none ? -INFINITY : (v - top) - logf(sum);
        e.mass = e.total = none ? 0.0f : sum >= 0.0f ? 1.0f : NAN;
    }
    return e;
}

// The listed elements of a row, one bit each: bit of element j at j - head + 8, so that a vector's bits lie in one word.
__host__ __device__ constexpr int list_words(int vocab) { return (vocab + 8 + 31) / 32 + 1; }
template <int DT>
__device__ __forceinline__ void note_listed(uint32_t *bits, const Row<DT> &row, int j)
{
    const int bit = j - row.head + 8;
    atomicOr(&bits[bit >> 5], 1u << (bit & 31));
}
template <int DT>
__device__ __forceinline__ bool is_listed(const uint32_t *bits, const Row<DT> &row, int j)
{
    const int bit = j - row.head + 8;
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
template <int DT>
__device__ __forceinline__ void hide_listed(const uint32_t *bits, const Row<DT> &row, int v, uint4 &raw)
{
    constexpr int kVec = Row<DT>::kVec;
    if (v >= row.vecs) return;
    const int bit = v * kVec + 8;
    const uint32_t hidden = (bits[bit >> 5] >> (bit & 31)) & ((1u << kVec) - 1u);
    if (hidden) hide_bits<DT>(hidden, raw);
}

template <int DT>
__global__ void __launch_bounds__(kLossThreads) distill_kernel(const Logits p, const TeacherList l, float *loss, float *saved)
{
    extern __shared__ __align__(16) uint32_t listed_bits[];
    __shared__ ListShared sh;
    __shared__ Sums part[2][kLossWarps];
    __shared__ float terms[kLossWarps];
    const int64_t r = blockIdx.x;
    const Row<DT> row(p.x, r * p.ld, p.vocab);
    for (int i = threadIdx.x; i < list_words(p.vocab); i += kLossThreads) listed_bits[i] = 0u;
    ListEntry e = load_list(p, l, r, sh);   // (has barriers behind the zeros)
    const bool counts = e.j >= 0;
    float x = -INFINITY;
    if (counts) {
        note_listed<DT>(listed_bits, row, e.j);
        x = row.at(e.j);
    }
    __syncthreads();
    // the tokens that are not listed, apart from those that are: neither sum is a difference
    Sums sums = {-INFINITY, 0.0f, 0.0f};
    stream_row<DT, false>(row, p.c, sums, [&](int v, uint4 &raw) { hide_listed<DT>(listed_bits, row, v, raw); });
    const int edge = row.edge(threadIdx.x);
    if (edge >= 0 && !is_listed<DT>(listed_bits, row, edge)) {
        const float y = row.at(edge);
        if (y > sums.m) sums.raise(y, p.c);
        sums.add<false>(y, p.c);
    }
    const Sums others = block_join(sums, p.c, part[0]);
    Sums own = {x, 0.0f, 0.0f};
    if (counts) own.add<false>(x, p.c);
    Sums all = block_join(own, p.c, part[1]);
    all.join(others, p.c);
    const bool none = all.s == 0.0f;
    const float logsum = none ? -INFINITY : logf(all.s);
    // ln of the others' sum relative to the row's largest logit, from the sum relative to their own: it may be far below
    const float logrest = others.s == 0.0f ? -INFINITY : __fmaf_rn(p.scale, others.m - all.m, logf(others.s));
    if (logrest == -INFINITY) e.drop_rest();
    float term = 0.0f;
    if (counts && e.q != 0.0f) term = e.q * (e.lnq - (none || x == -INFINITY ? -INFINITY : p.scale * (x - all.m) - logsum));
    if (threadIdx.x == 0 && e.rest != 0.0f) term += e.rest * (logf(e.rest) - (logrest - logsum));
    if (none && e.total != 0.0f && threadIdx.x == 0) term = INFINITY;
    term = block_sum<kLossThreads>(term, terms);
    if (threadIdx.x == 0) {
        loss[r] = term;
        if (saved)
            reinterpret_cast<float4 *>(saved)[r] = make_float4(none ? 0.0f : all.m, none ? INFINITY : logsum, 0.0f, none ? INFINITY : logrest);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------------------------------
struct GradOut {
    void *dx;
    int64_t ld;
    int same;   // rows of logits and gradient lie alike relative to 16 bytes
    AmaxSink sink;
};

// dx_j = 2^d (a + b d) with d = log2 p_j (p relative to the sum that log2sum is of), for all j of a row
// that `hide(v, vector)` leaves (the others are written as zeros, and later by their own formula); `skip(j)` is the same
// for elements outside the vectors
template <int DT, bool SLOPE, typename Hide, typename Skip>
__device__ __forceinline__ void write_row(const Row<DT> &row, void *out, int64_t at, int same, float m, float c, float log2sum, float a,
                                          float b, uint32_t &key, Hide hide, Skip skip)
{
    constexpr int kVec = Row<DT>::kVec, kUnroll = 4, kSize = InType<DT>::kBytes;
    auto value = [&](float x) {
        const float d = max_nan(__fmaf_rn(x - m, c, -log2sum), kFloor), e = exp2_approx(d);
        const uint32_t bits = element_bits<DT>(e * (SLOPE ? __fmaf_rn(b, d, a) : a));
        key = max(key, magnitude_key(element_value<DT>(bits)));
        return bits;
    };
    if (same) {
        uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(out) + (at + row.head) * kSize);
        for (int v0 = threadIdx.x; v0 < row.vecs; v0 += kUnroll * kLossThreads) {
            uint4 raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (v0 + u * kLossThreads < row.vecs) raw[u] = row.vectors()[v0 + u * kLossThreads];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (v0 + u * kLossThreads >= row.vecs) continue;
                float f[kVec];
                uint32_t w[4];
                hide(v0 + u * kLossThreads, raw[u]);
                unpack_vector<DT>(raw[u], f);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = DT == FP8_F32 ? value(f[i]) : value(f[2 * i % kVec]) | (value(f[(2 * i + 1) % kVec]) << 16);
                dst[v0 + u * kLossThreads] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        const int edge = row.edge(threadIdx.x);
        if (edge >= 0 && !skip(edge)) store_bits<DT>(out, at + edge, value(row.at(edge)));
    } else {
        for (int j = threadIdx.x; j < row.n; j += kLossThreads)
            if (!skip(j)) store_bits<DT>(out, at + j, value(row.at(j)));
    }
}

template <int DT>
__device__ __forceinline__ void write_zeros(void *out, int64_t at, int n)
{
    for (int j = threadIdx.x; j < n; j += kLossThreads) store_bits<DT>(out, at + j, 0u);
}

template <int DT>
__global__ void __launch_bounds__(kLossThreads) token_logprobs_bwd_kernel(const Logits p, const void *targets, const float *saved,
                                                                          const float *g_lp, int64_t g_lp_stride, const float *g_h,
                                                                          int64_t g_h_stride, const GradOut o)
{
    const int64_t r = blockIdx.x, at = r * o.ld;
    const float4 keep = reinterpret_cast<const float4 *>(saved)[r];
    int64_t t = g_lp && targets ? load_index(targets, p.it, r) : -1;
    if (t >= p.vocab) {
        if (threadIdx.x == 0) raise_flags(p.d_status, FP8_FLAG_BAD_INDEX);
        t = -1;
    }
    const float g = t >= 0 ? g_lp[r * g_lp_stride] : 0.0f, gh = g_h ? g_h[r * g_h_stride] : 0.0f;
    uint32_t key = 0;
    if ((g == 0.0f && gh == 0.0f) || keep.y == INFINITY) {
        write_zeros<DT>(o.dx, at, p.vocab);
    } else {
        const Row<DT> row(p.x, r * p.ld, p.vocab);
        uint32_t own = 0;
        if (t >= 0 && threadIdx.x == 0) {
            // 1 - p of a token that is nearly certain: expm1 keeps its digits
            const float lp = max_nan(p.scale * (row.at((int)t) - keep.x) - keep.y, -1e30f), prob = expf(lp);
            own = element_bits<DT>(p.scale * (-g * expm1f(lp) - gh * prob * (lp + keep.z)));
        }
        __syncthreads();   // (the gradient may overwrite the logits)
        write_row<DT, true>(row, o.dx, at, o.same, keep.x, p.c, keep.y * kLog2e, p.scale * (-g - gh * keep.z), -p.scale * gh * kLn2, key,
                            [&](int v, uint4 &raw) {
                                const int i = (int)t - row.head - v * Row<DT>::kVec;
                                if ((unsigned)i < (unsigned)Row<DT>::kVec) hide_bits<DT>(1u << i, raw);
                            },
                            [&](int j) { return j == (int)t; });
        __syncthreads();
        if (t >= 0 && threadIdx.x == 0) {
            store_bits<DT>(o.dx, at + t, own);
            key = max(key, magnitude_key(element_value<DT>(own)));
        }
    }
    sink_amax(key, o.sink);
}

template <int DT>
__global__ void __launch_bounds__(kLossThreads) distill_bwd_kernel(const Logits p, const TeacherList l, const float *saved,
                                                                   const float *g_loss, int64_t g_stride, const GradOut o)
{
    extern __shared__ __align__(16) uint32_t listed_bits[];
    __shared__ ListShared sh;
    const int64_t r = blockIdx.x, at = r * o.ld;
    const float4 keep = reinterpret_cast<const float4 *>(saved)[r];
    const float g = g_loss[r * g_stride] * p.scale;
    uint32_t key = 0;
    if (g == 0.0f || keep.y == INFINITY) {
        write_zeros<DT>(o.dx, at, p.vocab);
    } else {
        const Row<DT> row(p.x, r * p.ld, p.vocab);
        for (int i = threadIdx.x; i < list_words(p.vocab); i += kLossThreads) listed_bits[i] = 0u;
        ListEntry e = load_list(p, l, r, sh);   // (has barriers behind the zeros)
        if (keep.w == -INFINITY) e.drop_rest();
        uint32_t own = 0;
        if (e.j >= 0) {
            note_listed<DT>(listed_bits, row, e.j);
            const float prob = expf(p.scale * (row.at(e.j) - keep.x) - keep.y);
            own = element_bits<DT>(g * __fmaf_rn(e.total, prob, -e.q));
        }
        // the others: p_j Q, or with s_j = p_j / p_r, s_j (Q p_r - q_r): s_j is one of a sum of 1 however small p_r is
        const float logsum = e.rest == 0.0f ? keep.y : keep.w;
        const float a = e.rest == 0.0f ? e.total : __fmaf_rn(e.total, expf(keep.w - keep.y), -e.rest);
        __syncthreads();   // (the gradient may overwrite the logits)
        write_row<DT, false>(row, o.dx, at, o.same, keep.x, p.c, logsum * kLog2e, g * a, 0.0f, key,
                             [&](int v, uint4 &raw) { hide_listed<DT>(listed_bits, row, v, raw); },
                             [&](int j) { return is_listed<DT>(listed_bits, row, j); });
        __syncthreads();
        if (e.j >= 0) {
            store_bits<DT>(o.dx, at + e.j, own);
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

static GradOut make_grad(fp8_ctx *ctx, const void *x, int64_t ld, int dt, void *dx, int64_t ld_d, float *d_amax)
{
    const int64_t size = dt == FP8_F32 ? 4 : 2;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(x) & 15u) - (int64_t)(reinterpret_cast<uintptr_t>(dx) & 15u);
    const int same = apart == 0 && (ld - ld_d) * size % 16 == 0;
    return GradOut{dx, ld_d, same, {d_amax ? take_slot(ctx) : nullptr, d_amax, nullptr, ctx->d_status, FP8_E5, 0, 0}};
}

template <int DT>
static cudaError_t allow_lists()
{
    const int bytes = list_words(FP8_LOSS_VOCAB_MAX) * 4;
    cudaError_t e = cudaFuncSetAttribute(distill_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(distill_bwd_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e;
}
cudaError_t configure_loss_kernels()
{
    cudaError_t e = allow_lists<FP8_BF16>();
    if (e == cudaSuccess) e = allow_lists<FP8_F16>();
    return e == cudaSuccess ? allow_lists<FP8_F32>() : e;
}

}  // namespace fp8lin

#define FP8LIN_LAUNCH_BY_TYPE(KERNEL, GRID, SMEM, ...)                                                       \
    do {                                                                                                     \
        count_launch();                                                                                      \
        if (dt == FP8_BF16) KERNEL<FP8_BF16><<<GRID, kLossThreads, SMEM, (cudaStream_t)stream>>>(__VA_ARGS__);    \
        else if (dt == FP8_F16) KERNEL<FP8_F16><<<GRID, kLossThreads, SMEM, (cudaStream_t)stream>>>(__VA_ARGS__); \
        else KERNEL<FP8_F32><<<GRID, kLossThreads, SMEM, (cudaStream_t)stream>>>(__VA_ARGS__);                    \
    } while (0)

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
    FP8LIN_LAUNCH_BY_TYPE(token_logprobs_kernel, (unsigned)rows, 0, p, o);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
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
    if (!index_aligned(targets, (int)it) || !saved_aligned(saved) || !float_aligned(g_logprob) || !float_aligned(g_entropy) ||
        !element_aligned(dlogits, (int)dt) || !float_aligned(d_amax))
        return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const GradOut o = make_grad(ctx, logits, ld, (int)dt, dlogits, ld_d, d_amax);
    FP8LIN_LAUNCH_BY_TYPE(token_logprobs_bwd_kernel, (unsigned)rows, 0, p, targets, saved, g_logprob, g_logprob_stride, g_entropy,
                          g_entropy_stride, o);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
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
    FP8LIN_LAUNCH_BY_TYPE(distill_kernel, (unsigned)rows, list_words((int)vocab) * 4, p, l, loss, saved);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
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
    if (vocab > FP8_LOSS_VOCAB_MAX) return FP8_ERR_UNSUPPORTED;
    if (!saved_aligned(saved) || !float_aligned(g_loss) || !element_aligned(dlogits, (int)dt) || !float_aligned(d_amax)) return FP8_ERR_ALIGN;
    const OnDevice on(ctx->device);
    const Logits p = make_logits(ctx, logits, ld, rows, vocab, scale, (int)it);
    const TeacherList l = {index, value, ld_index, ld_value, listed, mode == FP8_DISTILL_REST};
    const GradOut o = make_grad(ctx, logits, ld, (int)dt, dlogits, ld_d, d_amax);
    FP8LIN_LAUNCH_BY_TYPE(distill_bwd_kernel, (unsigned)rows, list_words((int)vocab) * 4, p, l, saved, g_loss, g_loss_stride, o);
    return cudaGetLastError() == cudaSuccess ? FP8_OK : FP8_ERR_CUDA;
}

}  // extern "C"
