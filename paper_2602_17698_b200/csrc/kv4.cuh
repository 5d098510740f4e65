// The 4-bit key/value cache: layout and argument checks.
#pragma once
#include "fp4.cuh"
#include "kv8.cuh"

__host__ __device__ inline int kv4_code_pitch(int dim) { return (dim + 31) / 32 * 16; }      // bytes of a row
__host__ __device__ inline int kv4_scale_pitch(int dim) { return (dim + 63) / 64 * 4; }

inline int64_t kv4_table_pages(const sb_kv4_cache* c) { return c->table_pages ? c->table_pages : c->table_stride; }
// host checks shared by the calls on a cache
inline sb_status kv4_check(sb_ctx* ctx, const char* what, const sb_kv4_cache* c, int64_t total, const int32_t* starts,
                           const int32_t* lens, int64_t max_new) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !starts || !lens)
        return sb_fail(ctx, SB_ERR_INVALID, "%s: null", what);
    if (c->requests <= 0 || c->heads <= 0 || c->pages <= 0 || c->table_stride < 0 || c->table_pages < 0 || kv4_table_pages(c) <= 0 || total < 0 || max_new < 0)
        return sb_fail(ctx, SB_ERR_INVALID, "%s: empty cache or negative sizes", what);
    if (c->page_tokens <= 0 || c->page_tokens % SB_KV8_BLOCK || c->dim <= 0 || c->dim % 16 || c->dim > 256)
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: page_tokens a multiple of 16 and dim a multiple of 16 up to 256", what);
    if (c->requests > 65535 || c->heads > 65535 || c->pages >= (1ll << 31) || total >= (1ll << 31) || max_new >= (1ll << 31) ||
        kv4_table_pages(c) > ((1ll << 31) - 1) / c->page_tokens)
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: at most 65535 requests and heads, and 2^31 pages, rows and tokens of a request", what);
    if (!kv8_aligned16(c->k) || !kv8_aligned16(c->v) || !kv8_aligned16(c->k_scale) || !kv8_aligned16(c->v_scale) ||
        ((reinterpret_cast<uintptr_t>(c->k_head) | reinterpret_cast<uintptr_t>(c->v_head)) & 3))
        return sb_fail(ctx, SB_ERR_SHAPE, "%s: 16-byte aligned codes and scales", what);
    return SB_OK;
}
inline Kv8Geom kv4_geom(const sb_kv4_cache* c, int64_t total, const int32_t* starts, const int32_t* lens, int64_t max_new) {
    Kv8Geom g;
    g.table = c->table; g.table_stride = c->table_stride; g.pages = c->pages;
    g.requests = c->requests; g.heads = c->heads; g.page_tokens = c->page_tokens; g.dim = c->dim;
    g.starts = starts; g.lens = lens; g.total = total; g.max_new = (int)max_new;
    g.page = KvDiv(c->page_tokens); g.family = SBK_KV4;
    g.most = (int)std::min(kv4_table_pages(c) * c->page_tokens, KV_MOST);
    return g;
}
