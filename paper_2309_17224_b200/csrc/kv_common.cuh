// What the kernels on the paged FP8 cache share: argument checks, the walk from a row to its sequence and page.
#pragma once

#include "cast_common.cuh"
#include "fp8_kv.h"

namespace fp8lin {

inline bool kv_aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Checks of the cache and batch descriptors that every entry point makes.
inline fp8_status_t check_kv(const fp8_ctx *ctx, const fp8_kv_cache_t *c, const fp8_seq_batch_t *b, int conv)
{
    if (!ctx || !c || !b) return FP8_ERR_NULL;
    if (!c->k8 || !c->v8 || !c->bk || !c->bv || !b->d_q_start || !b->d_kv_len || !b->d_page_table) return FP8_ERR_NULL;
    if (conv < 0 || conv > 1) return FP8_ERR_DTYPE;
    if (c->pages <= 0 || c->kv_heads <= 0 || c->page_size <= 0 || c->head_dim <= 0) return FP8_ERR_SHAPE;
    if (b->seqs <= 0 || b->tokens <= 0 || b->max_q_len <= 0 || b->max_kv_len <= 0) return FP8_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return FP8_ERR_UNSUPPORTED;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return FP8_ERR_UNSUPPORTED;
    const int64_t slots = (int64_t)c->pages * c->page_size;
    if (slots >= (int64_t)1 << 31) return FP8_ERR_SHAPE;
    const int64_t page_biases = (int64_t)c->kv_heads * c->page_size;
    if (c->page_stride < page_biases * c->head_dim || c->bias_stride < page_biases) return FP8_ERR_SHAPE;
    if (b->table_stride < ((int64_t)b->max_kv_len + c->page_size - 1) / c->page_size) return FP8_ERR_SHAPE;
    if (!kv_aligned16(c->k8) || !kv_aligned16(c->v8) || !kv_aligned16(c->bk) || !kv_aligned16(c->bv) ||
        (c->page_stride % 16) != 0 || (c->bias_stride % 16) != 0)
        return FP8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(b->d_q_start) | reinterpret_cast<uintptr_t>(b->d_kv_len) |
         reinterpret_cast<uintptr_t>(b->d_page_table)) & 3u)
        return FP8_ERR_ALIGN;
    return FP8_OK;
}

// The descriptors as a kernel needs them (page_size is a power of two).
struct KvParams {
    uint8_t *k8, *v8;
    int8_t *bk, *bv;
    int64_t page_stride, bias_stride, table_stride;
    const int32_t *q_start, *kv_len, *table;
    int32_t pages, kv_heads, page_shift, seqs, tokens, max_q_len, max_kv_len;
    int32_t conv, delta;
    unsigned *d_status;
};
inline KvParams make_kv_params(const fp8_ctx *ctx, const fp8_kv_cache_t *c, const fp8_seq_batch_t *b, int conv)
{
    KvParams p;
    p.k8 = c->k8; p.v8 = c->v8; p.bk = c->bk; p.bv = c->bv;
    p.page_stride = c->page_stride; p.bias_stride = c->bias_stride; p.table_stride = b->table_stride;
    p.q_start = b->d_q_start; p.kv_len = b->d_kv_len; p.table = b->d_page_table;
    p.pages = c->pages; p.kv_heads = c->kv_heads; p.page_shift = __builtin_ctz((unsigned)c->page_size);
    p.seqs = b->seqs; p.tokens = b->tokens; p.max_q_len = b->max_q_len; p.max_kv_len = b->max_kv_len;
    p.conv = conv; p.delta = format_delta(FP8_E4, conv);
    p.d_status = ctx->d_status;
    return p;
}

#ifdef __CUDACC__

// Raise sticky bits, without an atomic where they stand already (a call can meet a condition in every row).
__device__ __forceinline__ void raise_flags(unsigned *d_status, unsigned bits)
{
    if (bits & ~*reinterpret_cast<volatile unsigned *>(d_status)) atomicOr(d_status, bits);
}

// The sequence that row t belongs to, found by the whole warp: the last b with q_start[b] <= t, thirty-two probes a
// round (one round up to 32 sequences).  -1 if t lies before the first or behind the last.
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ q_start, int seqs, int t, int lane)
{
    int lo = 0, hi = seqs;
    while (true) {
        const int step = (hi - lo + 31) >> 5, at = lo + lane * step;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, at < hi && __ldg(q_start + at) <= t));
        if (n == 0) return -1;
        lo += (n - 1) * step;
        hi = min(hi, lo + step);
        if (step == 1) break;
    }
    return t < __ldg(q_start + lo + 1) ? lo : -1;
}

// Where row t lies in the cache: page and place in the page.  Whole warp, uniform result.
//   kWritten: page and place are valid; kAbsent: position before the first token; kBad: outside the bounds
enum RowPlace { kWritten = 0, kAbsent = 1, kBad = 2 };
__device__ __forceinline__ RowPlace place_of_row(const KvParams &p, int t, int lane, int &page, int &off)
{
    const int b = find_sequence(p.q_start, p.seqs, t, lane);
    if (b < 0) return kBad;
    const int first = __ldg(p.q_start + b), n = __ldg(p.q_start + b + 1) - first, i = t - first;
    const int64_t pos = (int64_t)__ldg(p.kv_len + b) - n + i;
    if (pos < 0) return kAbsent;
    if (pos >= p.max_kv_len || i >= p.max_q_len) return kBad;
    page = __ldg(p.table + (int64_t)b * p.table_stride + (pos >> p.page_shift));
    off = (int)pos & ((1 << p.page_shift) - 1);
    return (unsigned)page < (unsigned)p.pages ? kWritten : kBad;
}

// 16 bytes that are used once.
__device__ __forceinline__ uint4 load_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// The bias that a cached row's bytes were cast under.
__device__ __forceinline__ int applied_bias(int b) { return b == FP8_KV_BIAS_NONFINITE ? 0 : b; }

#endif
}  // namespace fp8lin
