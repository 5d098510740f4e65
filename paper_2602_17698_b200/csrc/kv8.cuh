// The 8-bit key/value cache: layout, argument checks, conversions.
#pragma once
#include "common.cuh"

// Quotients of 31-bit numbers by a divisor that the host knows: with m = ceil(2^64 / d),
// floor(x m / 2^64) is exact while x and d are below 2^31 (d = 1: m does not fit, m = 0).
struct KvDiv {
    uint64_t m = 0;
    int d = 1;
    KvDiv() = default;
    explicit KvDiv(int d_) : m(d_ > 1 ? ~0ull / (unsigned)d_ + 1 : 0), d(d_) {}
#ifdef __CUDACC__
    __device__ __forceinline__ int quot(int x) const { return d > 1 ? (int)__umul64hi((unsigned long long)(unsigned)x, m) : x; }
    __device__ __forceinline__ int rem(int x) const { return x - quot(x) * d; }
#endif
};

struct Kv8Geom {                 // the parts of sb_kv8_cache that kernels read
    const int32_t* table;
    int64_t table_stride, pages;
    int requests, heads, page_tokens, dim;
    int most;                    // tokens a request may have: what its pages hold
    const int32_t* starts;
    const int32_t* lens;
    int64_t total;               // rows of the call's dense arguments
    int max_new;
    KvDiv page;                  // by page_tokens
};

inline bool kv8_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline int64_t kv8_table_pages(const sb_kv8_cache* c) { return c->table_pages ? c->table_pages : c->table_stride; }
// host checks shared by the calls on a cache
inline sb_status kv8_check(sb_ctx* ctx, const char* what, const sb_kv8_cache* c, int64_t total, const int32_t* starts,
                           const int32_t* lens, int64_t max_new) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !starts || !lens)
        return sb_fail(ctx, SB_ERR_INVALID, "%s: null", what);
    if (c->requests <= 0 || c->heads <= 0 || c->pages <= 0 || c->table_stride < 0 || kv8_table_pages(c) <= 0 || total < 0 || max_new < 0)
        return sb_fail(ctx, SB_ERR_INVALID, "%s: empty cache or negative sizes", what);
    if (c->type != SB_KV_INT8 && c->type != SB_KV_E4M3) return sb_fail(ctx, SB_ERR_INVALID, "%s: unknown type %d", what, c->type);
    if (c->page_tokens <= 0 || c->page_tokens % SB_KV8_BLOCK || c->dim <= 0 || c->dim % 16 || c->dim > 256)
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: page_tokens a multiple of 16 and dim a multiple of 16 up to 256", what);
    if (c->requests > 65535 || c->heads > 65535 || c->pages >= (1ll << 31) || total >= (1ll << 31) || max_new >= (1ll << 31) ||
        kv8_table_pages(c) > ((1ll << 31) - 1) / c->page_tokens)
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: at most 65535 requests and heads, and 2^31 pages, rows and tokens of a request", what);
    if (!kv8_aligned16(c->k) || !kv8_aligned16(c->v) || (reinterpret_cast<uintptr_t>(c->k_scale) & 1) || (reinterpret_cast<uintptr_t>(c->v_scale) & 1))
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: 16-byte aligned codes and 2-byte aligned scales", what);
    return SB_OK;
}
inline Kv8Geom kv8_geom(const sb_kv8_cache* c, int64_t total, const int32_t* starts, const int32_t* lens, int64_t max_new) {
    Kv8Geom g;
    g.table = c->table; g.table_stride = c->table_stride; g.pages = c->pages;
    g.requests = c->requests; g.heads = c->heads; g.page_tokens = c->page_tokens; g.dim = c->dim;
    g.starts = starts; g.lens = lens; g.total = total; g.max_new = (int)max_new;
    g.page = KvDiv(c->page_tokens);
    g.most = (int)(kv8_table_pages(c) * c->page_tokens);
    return g;
}

#ifdef __CUDACC__
struct Kv8Request { int row0, n, len, past; };      // first dense row, new tokens, tokens in the cache, of them earlier
// The request's numbers; false (and the status latched) where they do not fit the call.
__device__ __forceinline__ bool kv8_request(const Kv8Geom& g, int b, Kv8Request& r, SbDeviceState* st) {
    r.row0 = g.starts[b];
    const int64_t n = (int64_t)g.starts[b + 1] - r.row0;
    r.len = g.lens[b];
    r.n = (int)n;
    r.past = r.len - r.n;
    const bool ok = r.row0 >= 0 && n >= 0 && n <= g.max_new && r.row0 + n <= g.total && r.len >= n &&
                    r.len <= g.most;
    if (!ok) sb_latch(st, SB_ERR_INVALID, SBK_KV8);
    return ok;
}
// Page of a request's token block; false (and the status latched) where it lies outside the cache.
__device__ __forceinline__ bool kv8_page(const Kv8Geom& g, int b, int page_index, int64_t& page, SbDeviceState* st) {
    page = g.table[(int64_t)b * g.table_stride + page_index];
    if (page >= 0 && page < g.pages) return true;
    sb_latch(st, SB_ERR_INVALID, SBK_KV8);
    return false;
}

// pairs of codes (16 bits, the first in the low byte) to pairs of fp16, exact
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t pair) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)pair));
    return h;
}
#endif
