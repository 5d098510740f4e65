// Writing and reading the 4-bit key/value cache.
//
// A thread takes one block of 16 elements of a token's head, of the keys or of the values: 32 bytes in, 8 bytes of codes and a
// scale byte out. The scales of four blocks are four consecutive bytes: the lanes that hold them pass them to the
// first, which stores one word. Blocks are independent of one another, so writing needs no look at what the cache holds.
#include "kv4.cuh"
#include "launch.cuh"

namespace {

constexpr int K4_THREADS = 256;

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
        const float dd = d > 0.f ? d : 1.f, r = __frcp_rn(dd);       // d = 0: every code is 0
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = d > 0.f ? w[i] : 0u;
            v[i >> 2][2 * (i & 3)] = div_rn(bf16lo(x), dd, r);
            v[i >> 2][2 * (i & 3) + 1] = div_rn(bf16hi(x), dd, r);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = (i & 1) ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]);
            v[i >> 3][i & 7] = e != e ? 0.f : fabsf(e) > 3.4e38f ? copysignf(6.f, e) : d > 0.f ? __fdiv_rn(e, d) : 0.f;
        }
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
    const Kv4Side& sd = blockIdx.z ? vs : ks;
    // unit: (row, head, block), the block fastest; four lanes side by side hold four blocks of a row of scales
    const int64_t unit = (int64_t)blockIdx.x * K4_THREADS + threadIdx.x;
    const bool mine = unit < (int64_t)rq.n * per_row.d;
    const unsigned lanes = __ballot_sync(0xffffffffu, mine);
    if (!mine) return;
    const int i = per_row.quot((int)unit), rest = (int)unit - i * per_row.d;
    const int head = blocks.quot(rest), j = rest - head * blocks.d;
    const int tok = rq.past + i;
    const int64_t page = g.table[(int64_t)b * g.table_stride + g.page.quot(tok)];
    uint32_t w[8], scale = 0;
    uint2 codes = make_uint2(0, 0);
    const bool there = page >= 0 && page < g.pages;
    if (!there) sb_latch(st, SB_ERR_INVALID, SBK_KV8);
    if (16 * j < g.dim) {
        const __nv_bfloat16* x = sd.x + (int64_t)(rq.row0 + i) * sd.token_stride + (int64_t)head * sd.head_stride + 16 * j;
        const uint4 a = ld_stream16(x), c = ld_stream16(x + 8);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = c.x; w[5] = c.y; w[6] = c.z; w[7] = c.w;
        if (!kv4_codes(w, sd.head ? __ldg(sd.head + head) : 1.f, codes, scale)) sb_latch(st, SB_ERR_NONFINITE, SBK_KV8);
    }
    uint32_t word = scale;
    word |= __shfl_down_sync(lanes, scale, 1) << 8;
    word |= __shfl_down_sync(lanes, word, 2) << 16;
    if (!there) return;
    const int64_t at = (page * g.heads + head) * g.page_tokens + g.page.rem(tok);
    const int pitch = kv4_code_pitch(g.dim);
    if (8 * j < pitch) *reinterpret_cast<uint2*>(sd.codes + at * pitch + 8 * j) = codes;
    if ((j & 3) == 0) *reinterpret_cast<uint32_t*>(sd.scales + at * blocks.d + j) = word;
}

__global__ void __launch_bounds__(K4_THREADS)
kv4_read_kernel(const Kv8Geom g, const Kv4Side ks, const Kv4Side vs, const KvDiv per_row, const KvDiv blocks,
                __nv_bfloat16* __restrict__ K, __nv_bfloat16* __restrict__ V, SbDeviceState* st) {
    const int b = blockIdx.y;
    sb_let_next();
    sb_after_previous();
    Kv8Request rq;
    if (!kv8_request(g, b, rq, st)) return;
    const Kv4Side& sd = blockIdx.z ? vs : ks;
    const int64_t unit = (int64_t)blockIdx.x * K4_THREADS + threadIdx.x;           // (row, head, block)
    if (unit >= (int64_t)rq.n * per_row.d) return;
    const int i = per_row.quot((int)unit), rest = (int)unit - i * per_row.d;
    const int head = blocks.quot(rest), j = rest - head * blocks.d;
    const int tok = rq.past + i;
    int64_t page;
    if (!kv8_page(g, b, g.page.quot(tok), page, st)) return;
    const int64_t at = (page * g.heads + head) * g.page_tokens + g.page.rem(tok);
    const uint2 codes = *reinterpret_cast<const uint2*>(sd.codes + at * kv4_code_pitch(g.dim) + 8 * j);
    const float s = e4m3_value(sd.scales[at * kv4_scale_pitch(g.dim) + j]), h = sd.head ? __ldg(sd.head + head) : 1.f;
    uint32_t p[2][4], o[8];
    fp4_unpack8(codes.x, p[0]);
    fp4_unpack8(codes.y, p[1]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p[k >> 2][k & 3]));
        o[k] = u32(__floats2bfloat162_rn(f.x * s * h, f.y * s * h));              // code times scale is exact
    }
    __nv_bfloat16* y = (blockIdx.z ? V : K) + ((int64_t)(rq.row0 + i) * g.heads + head) * g.dim + 16 * j;
    *reinterpret_cast<uint4*>(y) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(y + 8) = make_uint4(o[4], o[5], o[6], o[7]);
}

// blocks of threads for max_new rows of `per_row` units; false: too many
bool kv4_grid(const sb_kv4_cache* c, int64_t max_new, int64_t per_row, dim3& grid) {
    const int64_t units = max_new * per_row;
    if (per_row >= (1ll << 31) || units >= (1ll << 31)) return false;
    grid = dim3((unsigned)((units + K4_THREADS - 1) / K4_THREADS), (unsigned)c->requests, 2);
    return true;
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
    if (!kv4_grid(cache, max_new, (int64_t)cache->heads * blocks, grid)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 append: max_new x heads too large");
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
    const int blocks = cache->dim / 16;
    dim3 grid;
    if (!kv4_grid(cache, max_new, (int64_t)cache->heads * blocks, grid)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 read: max_new x heads too large");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    const Kv4Side ks{static_cast<uint8_t*>(cache->k), static_cast<uint8_t*>(cache->k_scale), cache->k_head, nullptr, 0, 0};
    const Kv4Side vs{static_cast<uint8_t*>(cache->v), static_cast<uint8_t*>(cache->v_scale), cache->v_head, nullptr, 0, 0};
    return sb_launch(ctx, kv4_read_kernel, grid, K4_THREADS, 0, 1, true, kv4_geom(cache, total, starts, lens, max_new), ks, vs,
                     KvDiv(cache->heads * blocks), KvDiv(blocks), static_cast<__nv_bfloat16*>(K), static_cast<__nv_bfloat16*>(V), ctx->dstate);
}
