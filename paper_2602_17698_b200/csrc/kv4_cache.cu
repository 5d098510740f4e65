// Writing and reading the 4-bit key/value cache.
//
// A thread takes one block of 16 elements of a token's head, of the keys and of the values: 32 bytes in, 8 bytes of codes and a
// scale byte out, each. The scales of four blocks are four consecutive bytes: the lanes that hold them pass them to the
// first, which stores one word. Blocks are independent of one another, so writing needs no look at what the cache holds.
//
// Where there are many rows both are bound by issuing instructions (66 % of the slots while a multiprocessor is busy), most of which find
// a block's place and its rows: one thread for keys and values and packed quotients took 8000 rows of 8 heads of 128 from 16 us
// to 12.5, several rows a thread in reading from 10 to 7.5 (writing got slower by it: its rows are longer chains). Where there are few
// rows, the chain of dependent reads (request, table, codes) is all there is.
#include "kv4.cuh"
#include "launch.cuh"

namespace {

constexpr int K4_THREADS = 128;

struct Kv4Side {
    uint8_t *codes, *scales;
    const float* head;
    const __nv_bfloat16* x;
    int64_t token_stride, head_stride;
};

// Codes of 16 elements and the scale byte of their block; false: there was something not finite.
__device__ __forceinline__ bool kv4_codes(const uint32_t (&w)[8], float g, uint2& codes, uint32_t& scale) {
    codes = make_uint2(0, 0);
    scale = 0;
    if (!(g > 0.f) || g > 3.4e38f) return false;
    // the largest magnitude as bf16 bits, whose order is the order of the numbers
    uint32_t m2 = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m2 = __vmaxu2(m2, w[i] & 0x7fff7fffu);
    uint32_t amax = max(m2 & 0xffffu, m2 >> 16);
    const bool fine = amax < 0x7f80u;
    if (!fine) {
        amax = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t e = (w[i >> 1] >> (16 * (i & 1))) & 0x7fffu;
            if (e < 0x7f80u) amax = max(amax, e);
        }
    }
    const float am = __uint_as_float(amax << 16);
    // the quotients the short way where everything stays in range
    const bool near = g > 0x1p-50f && g < 0x1p30f && am > 0x1p-60f && am < 0x1p60f;
    const float t = near ? div_rn(div_rn(am, 6.f, 0.16666667f), g, __frcp_rn(g)) : __fdiv_rn(__fdiv_rn(am, 6.f), g);
    scale = e4m3_of(fminf(t, 448.f));
    const float d = e4m3_value(scale) * g;
    float v[2][8];
    if (fine && ((div_in_range(d) && t < 0x1p100f) || d == 0.f)) {
        // -x / d, two at a time: as div_rn with every sign turned, so that a zero's sign is kept; d = 0: every code is 0
        const float dd = d > 0.f ? d : 1.f, r = __frcp_rn(dd);
        const f32x2 d2 = pk2(dd, dd), r2 = pk2(-r, -r);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 x = pk2(bf16lo(w[i]), bf16hi(w[i])), q = mul2(x, r2);
            upk2(fma2(fma2(q, d2, x), r2, q), v[i >> 2][2 * (i & 3)], v[i >> 2][2 * (i & 3) + 1]);
        }
        const uint32_t turn = 0x88888888u;
        codes = d > 0.f ? make_uint2(fp4_pack8(v[0]) ^ turn, fp4_pack8(v[1]) ^ turn) : make_uint2(0, 0);
        return true;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float e = (i & 1) ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]);
        v[i >> 3][i & 7] = e != e ? 0.f : fabsf(e) > 3.4e38f ? copysignf(6.f, e) : d > 0.f ? __fdiv_rn(e, d) : 0.f;
    }
    codes = make_uint2(fp4_pack8(v[0]), fp4_pack8(v[1]));
    return fine;
}

__global__ void __launch_bounds__(K4_THREADS)
kv4_append_kernel(const Kv8Geom g, const Kv4Side ks, const Kv4Side vs, const KvDiv per_row, const KvDiv blocks, SbDeviceState* st) {
    const int b = blockIdx.y;
    sb_let_next();
    sb_after_previous();
    Kv8Request rq;
    if (!kv8_request(g, b, rq, st)) return;
    // unit: (row, head, block), the block fastest; four lanes side by side hold four blocks of a row of scales
    const int64_t unit = (int64_t)blockIdx.x * K4_THREADS + threadIdx.x;
    if (unit >= (int64_t)rq.n * per_row.d) return;
    const unsigned four = 15u << (threadIdx.x & 28);
    const int i = per_row.quot((int)unit), rest = (int)unit - i * per_row.d;
    const int head = blocks.quot(rest), j = rest - head * blocks.d;
    const int tok = rq.past + i;
    const int64_t page = g.table[(int64_t)b * g.table_stride + g.page.quot(tok)];
    const bool inside = 16 * j < g.dim;
    uint32_t w[2][8];
    float by[2];
    if (inside) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Kv4Side& sd = k ? vs : ks;
            const __nv_bfloat16* x = sd.x + (int64_t)(rq.row0 + i) * sd.token_stride + (int64_t)head * sd.head_stride + 16 * j;
            const uint4 a = ld_once16(x), c = ld_once16(x + 8);
            w[k][0] = a.x; w[k][1] = a.y; w[k][2] = a.z; w[k][3] = a.w;
            w[k][4] = c.x; w[k][5] = c.y; w[k][6] = c.z; w[k][7] = c.w;
            by[k] = sd.head ? sd.head[head] : 1.f;
        }
    }
    const bool there = page >= 0 && page < g.pages;
    if (!there) sb_latch(st, SB_ERR_INVALID, SBK_KV4);
    const int64_t at = (page * g.heads + head) * g.page_tokens + g.page.rem(tok);
    const int pitch = kv4_code_pitch(g.dim);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const Kv4Side& sd = k ? vs : ks;
        uint32_t scale = 0;
        uint2 codes = make_uint2(0, 0);
        if (inside && !kv4_codes(w[k], by[k], codes, scale)) sb_latch(st, SB_ERR_NONFINITE, SBK_KV4);
        uint32_t word = scale;
        word |= __shfl_down_sync(four, scale, 1) << 8;
        word |= __shfl_down_sync(four, word, 2) << 16;
        if (!there) continue;
        if (8 * j < pitch) *reinterpret_cast<uint2*>(sd.codes + at * pitch + 8 * j) = codes;
        if ((j & 3) == 0) *reinterpret_cast<uint32_t*>(sd.scales + at * blocks.d + j) = word;
    }
}

// Where a request's token lies, token by token
struct Kv4Walk {
    int slot, entry;
    int64_t page;
    __device__ __forceinline__ void find(const Kv8Geom& g, int b) { page = g.table[(int64_t)b * g.table_stride + entry]; }
    __device__ __forceinline__ void begin(const Kv8Geom& g, int b, int tok) {
        entry = g.page.quot(tok);
        slot = tok - entry * g.page_tokens;
        find(g, b);
    }
    __device__ __forceinline__ void next(const Kv8Geom& g, int b) {
        if (++slot < g.page_tokens) return;
        slot = 0;
        ++entry;
        find(g, b);
    }
    __device__ __forceinline__ bool there(const Kv8Geom& g) const { return page >= 0 && page < g.pages; }
    __device__ __forceinline__ int64_t at(const Kv8Geom& g, int head) const { return (page * g.heads + head) * g.page_tokens + slot; }
};

// ROWS: of a thread, so that what it finds out first pays for several
template <int ROWS>
__global__ void __launch_bounds__(K4_THREADS)
kv4_read_kernel(const Kv8Geom g, const Kv4Side ks, const Kv4Side vs, const KvDiv per_row, const KvDiv blocks,
                __nv_bfloat16* __restrict__ K, __nv_bfloat16* __restrict__ V, SbDeviceState* st) {
    const int b = blockIdx.y;
    sb_let_next();
    sb_after_previous();
    Kv8Request rq;
    if (!kv8_request(g, b, rq, st)) return;
    const int64_t unit = (int64_t)blockIdx.x * K4_THREADS + threadIdx.x;           // (rows, head, half a block): a warp's stores are side by side
    if (unit >= (int64_t)((rq.n + ROWS - 1) / ROWS) * per_row.d) return;
    const int group = per_row.quot((int)unit), rest = (int)unit - group * per_row.d;
    const int head = blocks.quot(rest), j = rest - head * blocks.d;
    const int pitch = kv4_code_pitch(g.dim), spitch = kv4_scale_pitch(g.dim);
    Kv4Walk walk;
    walk.begin(g, b, rq.past + ROWS * group);
    const float by[2] = {ks.head ? ks.head[head] : 1.f, vs.head ? vs.head[head] : 1.f};
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int i = ROWS * group + r;
        if (i >= rq.n) break;
        if (r > 0) walk.next(g, b);
        if (!walk.there(g)) {
            sb_latch(st, SB_ERR_INVALID, SBK_KV4);
            continue;
        }
        const int64_t at = walk.at(g, head), to = ((int64_t)(rq.row0 + i) * g.heads + head) * g.dim + 8 * j;
        uint32_t codes[2], scale[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Kv4Side& sd = k ? vs : ks;
            codes[k] = *reinterpret_cast<const uint32_t*>(sd.codes + at * pitch + 4 * j);
            scale[k] = sd.scales[at * spitch + (j >> 1)];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t s2 = e4m3x2_to_f16x2(scale[k] | scale[k] << 8);
            const f32x2 h2 = pk2(by[k], by[k]);
            uint32_t p[4], o[4];
            fp4_unpack8(codes[k], p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = f16x2_mul(p[e], s2);                   // code times scale is exact
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
                float lo, hi;
                upk2(mul2(pk2(f.x, f.y), h2), lo, hi);
                o[e] = u32(__floats2bfloat162_rn(lo, hi));
            }
            *reinterpret_cast<uint4*>((k ? V : K) + to) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// blocks of threads for max_new rows of `per_row` units, `rows` of a thread; false: too many
bool kv4_grid(const sb_kv4_cache* c, int64_t max_new, int rows, int64_t per_row, dim3& grid) {
    const int64_t units = (max_new + rows - 1) / rows * per_row;
    if (per_row >= (1ll << 31) || max_new * per_row >= (1ll << 31)) return false;
    grid = dim3((unsigned)((units + K4_THREADS - 1) / K4_THREADS), (unsigned)c->requests);
    return true;
}

// Rows of a thread: what a thread finds out first pays for several where there are enough of them (8 warps a scheduler all the same).
int kv4_rows(const sb_ctx* ctx, const sb_kv4_cache* c, int64_t total, int blocks) {
    return total * c->heads * blocks >= (int64_t)ctx->sm_count * 1024 * 4 ? 4 : 1;
}

}  // namespace

extern "C" sb_status sb_kv4_append(sb_ctx* ctx, const sb_kv4_cache* cache, const void* K, int64_t k_token_stride,
                                   int64_t k_head_stride, const void* V, int64_t v_token_stride, int64_t v_head_stride,
                                   int64_t total, const int32_t* starts, const int32_t* lens, int64_t max_new) {
    if (!ctx) return SB_ERR_INVALID;
    const sb_status s = kv4_check(ctx, "kv4 append", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!K || !V) return sb_fail(ctx, SB_ERR_INVALID, "kv4 append: null");
    if (!kv8_aligned16(K) || !kv8_aligned16(V) || k_token_stride % 8 || k_head_stride % 8 || v_token_stride % 8 || v_head_stride % 8)
        return sb_fail(ctx, SB_ERR_SHAPE, "kv4 append: strides that are multiples of 8 and 16-byte aligned bases");
    const int blocks = kv4_scale_pitch(cache->dim);
    dim3 grid;
    if (!kv4_grid(cache, max_new, 1, (int64_t)cache->heads * blocks, grid)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 append: max_new x heads too large");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    const Kv4Side ks{static_cast<uint8_t*>(cache->k), static_cast<uint8_t*>(cache->k_scale), cache->k_head,
                     static_cast<const __nv_bfloat16*>(K), k_token_stride, k_head_stride};
    const Kv4Side vs{static_cast<uint8_t*>(cache->v), static_cast<uint8_t*>(cache->v_scale), cache->v_head,
                     static_cast<const __nv_bfloat16*>(V), v_token_stride, v_head_stride};
    return sb_launch(ctx, kv4_append_kernel, grid, K4_THREADS, 0, 1, true, kv4_geom(cache, total, starts, lens, max_new), ks, vs,
                     KvDiv(cache->heads * blocks), KvDiv(blocks), ctx->dstate);
}

extern "C" sb_status sb_kv4_read(sb_ctx* ctx, const sb_kv4_cache* cache, int64_t total, const int32_t* starts,
                                 const int32_t* lens, int64_t max_new, void* K, void* V) {
    if (!ctx) return SB_ERR_INVALID;
    const sb_status s = kv4_check(ctx, "kv4 read", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!K || !V || K == V) return sb_fail(ctx, SB_ERR_INVALID, "kv4 read: null, or one output for both");
    if (!kv8_aligned16(K) || !kv8_aligned16(V)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 read: 16-byte aligned outputs");
    const int blocks = cache->dim / 8;
    dim3 grid;
    const int rows = kv4_rows(ctx, cache, total, blocks);
    if (!kv4_grid(cache, max_new, rows, (int64_t)cache->heads * blocks, grid)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 read: max_new x heads too large");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    const Kv4Side ks{static_cast<uint8_t*>(cache->k), static_cast<uint8_t*>(cache->k_scale), cache->k_head, nullptr, 0, 0};
    const Kv4Side vs{static_cast<uint8_t*>(cache->v), static_cast<uint8_t*>(cache->v_scale), cache->v_head, nullptr, 0, 0};
    return sb_launch(ctx, rows == 1 ? kv4_read_kernel<1> : kv4_read_kernel<4>, grid, K4_THREADS, 0, 1, true, kv4_geom(cache, total, starts, lens, max_new), ks, vs,
                     KvDiv(cache->heads * blocks), KvDiv(blocks), static_cast<__nv_bfloat16*>(K), static_cast<__nv_bfloat16*>(V), ctx->dstate);
}
