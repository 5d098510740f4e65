// Writing and reading the 8-bit key/value cache.
//
// A warp owns one scale block: the 16 tokens x dim codes of one head that share a scale, of the
// keys or of the values. It reads what the block already holds of the request and what the call
// brings, reduces the new tokens' largest magnitude, and writes codes and scale: no other warp
// touches them, so nothing has to be ordered between warps, and the kernel needs one pass. An
// element costs 2 bytes read and 1 written; earlier tokens are only rewritten when the scale grew.
// 6 requests of up to 2048 tokens, 8 heads of 128, written and read back: 29 us, 3.4 TB/s; issue bounds
// it (56 and 67 % of the slots): exact quotients, conversions. 64 x 1 token: 8.3 us, two launches.
#include "kv8.cuh"

namespace {

constexpr int KA_WARPS = 4;

struct KvSide {
    uint8_t* codes;
    uint16_t* scale;
    const __nv_bfloat16* x;
    int64_t token_stride, head_stride;
};

// smallest bf16 not below x (x >= 0, finite), as its bits
__device__ __forceinline__ uint32_t bf16_up(float x) {
    const uint32_t u = __float_as_uint(x);
    return (u + 0xffffu) >> 16;
}

// eight fp32 values within the type's range to eight codes
template <int TYPE>
__device__ __forceinline__ uint2 to_codes(const float (&v)[8]) {
    uint32_t w[2];
    if (TYPE == SB_KV_INT8) {
        // 1.5 * 2^23 rounds to a whole number (nearest, ties to even) and leaves it in the low byte
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(v[i] + 12582912.f);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            w[h] = __byte_perm(__byte_perm(b[4 * h], b[4 * h + 1], 0x0040), __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040), 0x5410);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            asm("{\n\t.reg .b16 a, b;\n\t"
                "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
                "mov.b32 %0, {a, b};\n\t}"
                : "=r"(w[h]) : "f"(v[4 * h]), "f"(v[4 * h + 1]), "f"(v[4 * h + 2]), "f"(v[4 * h + 3]));
    }
    return make_uint2(w[0], w[1]);
}
template <int TYPE>
__device__ __forceinline__ void from_codes(uint2 c, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t pair = ((i < 2 ? c.x : c.y) >> (16 * (i & 1))) & 0xffffu;
        if (TYPE == SB_KV_INT8) {
            v[2 * i] = (float)(int8_t)(pair & 0xff);
            v[2 * i + 1] = (float)(int8_t)(pair >> 8);
        } else {
            const uint32_t h = e4m3x2_to_f16x2(pair);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

// NC: 16-byte pieces of the block's new tokens a lane holds (dim / 16 of them are used)
template <int TYPE, int NC>
__global__ void __launch_bounds__(KA_WARPS * 32)
kv8_append_kernel(const Kv8Geom g, const KvSide ks, const KvSide vs, SbDeviceState* st) {
    const int lane = threadIdx.x & 31;
    const int b = blockIdx.y;
    Kv8Request rq;
    if (!kv8_request(g, b, rq, st) || rq.n == 0) return;
    const int blk0 = rq.past / SB_KV8_BLOCK;
    const int nblk = (rq.len + SB_KV8_BLOCK - 1) / SB_KV8_BLOCK - blk0;
    const int unit = blockIdx.x * KA_WARPS + (threadIdx.x >> 5);         // (block, head, side), the side fastest
    const int bi = unit / (2 * g.heads);
    if (bi >= nblk) return;
    const int head = (unit >> 1) % g.heads;
    const KvSide sd = (unit & 1) ? vs : ks;
    const int tok0 = (blk0 + bi) * SB_KV8_BLOCK;                         // first token of the block
    int64_t page;
    if (!kv8_page(g, b, g.page.quot(tok0), page, st)) return;
    const int slot = g.page.rem(tok0);
    const int64_t ph = page * g.heads + head;
    uint8_t* codes = sd.codes + (ph * g.page_tokens + slot) * g.dim;
    uint16_t* scale_at = sd.scale + ph * (g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK;

    const int per_tok = g.dim >> 3;                                      // pieces of 8 elements per token
    const int old_toks = max(0, min(SB_KV8_BLOCK, rq.past - tok0)), toks = min(SB_KV8_BLOCK, rq.len - tok0);
    uint4 x[NC];
    uint32_t m2 = 0;                                                     // largest magnitudes, as bf16 bits
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int piece = lane + 32 * i, tok = piece / per_tok;
        x[i] = make_uint4(0, 0, 0, 0);
        if (piece < SB_KV8_BLOCK * per_tok && tok >= old_toks && tok < toks) {
            const int64_t row = rq.row0 + (tok0 + tok - rq.past);
            x[i] = ld_stream16(sd.x + row * sd.token_stride + head * sd.head_stride + 8 * (piece - tok * per_tok));
        }
    }
    const uint32_t before = old_toks ? *scale_at : 0u;                   // non-negative: the bits are ordered as the numbers
#pragma unroll
    for (int i = 0; i < NC; ++i)
        m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
    uint32_t amax = __reduce_max_sync(0xffffffffu, max(m2 & 0xffffu, m2 >> 16));
    constexpr float QMAX = TYPE == SB_KV_INT8 ? 127.f : 448.f;
    const bool bad = amax >= 0x7f80u;
    if (bad) {
        // a NaN or an infinity: the scale is the finite elements'
        amax = 0;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t e = (w[k >> 1] >> (16 * (k & 1))) & 0x7fffu;
                if (e < 0x7f80u) amax = max(amax, e);
            }
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        if (lane == 0) sb_latch(st, SB_ERR_NONFINITE, SBK_KV8);
    }
    uint32_t sbits = bf16_up(__fdiv_rn(__uint_as_float(amax << 16), QMAX));
    const bool grew = sbits > before;
    if (!grew) sbits = before;
    const float s = __uint_as_float(sbits << 16), s_old = __uint_as_float(before << 16);
    const bool quick = div_in_range(s) && !bad;
    const float rs = quick ? __frcp_rn(s) : 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int piece = lane + 32 * i, tok = piece / per_tok;
        if (piece >= SB_KV8_BLOCK * per_tok || tok >= toks || (tok < old_toks && !grew)) continue;
        uint2* at = reinterpret_cast<uint2*>(codes + 8 * (int64_t)piece);
        float v[8];
        if (tok < old_toks) {
            from_codes<TYPE>(*at, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __fdiv_rn(v[k] * s_old, s);
        } else {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            if (quick) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = div_rn((k & 1) ? bf16hi(w[k >> 1]) : bf16lo(w[k >> 1]), s, rs);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float e = (k & 1) ? bf16hi(w[k >> 1]) : bf16lo(w[k >> 1]);
                    v[k] = e != e ? 0.f : fabsf(e) > 3.4e38f ? copysignf(QMAX, e) : s > 0.f ? __fdiv_rn(e, s) : 0.f;
                }
            }
        }
        *at = to_codes<TYPE>(v);
    }
    if (lane == 0 && (grew || !old_toks)) *scale_at = (uint16_t)sbits;
}

template <int TYPE>
__global__ void __launch_bounds__(256)
kv8_read_kernel(const Kv8Geom g, const KvSide ks, const KvSide vs, __nv_bfloat16* __restrict__ K,
                __nv_bfloat16* __restrict__ V, SbDeviceState* st) {
    const int b = blockIdx.y;
    Kv8Request rq;
    if (!kv8_request(g, b, rq, st)) return;
    const int per_tok = g.dim >> 3;                                      // pieces of 8 elements per token and head
    const int64_t per_row = (int64_t)g.heads * per_tok;
    const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;        // (row, head, piece), keys and values both
    if (unit >= rq.n * per_row) return;
    const int i = (int)(unit / per_row), rest = (int)(unit - i * per_row);
    const int head = rest / per_tok, piece = rest - head * per_tok;
    const int tok = rq.past + i;
    int64_t page;
    if (!kv8_page(g, b, g.page.quot(tok), page, st)) return;
    const int slot = g.page.rem(tok);
    const int64_t ph = page * g.heads + head;
    const int64_t src = (ph * g.page_tokens + slot) * g.dim + 8 * piece;
    const int64_t sat = ph * (g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK;
    const int64_t dst = ((int64_t)(rq.row0 + i) * g.heads + head) * g.dim + 8 * piece;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const KvSide& sd = side ? vs : ks;
        const float s = __uint_as_float((uint32_t)sd.scale[sat] << 16);
        float v[8];
        from_codes<TYPE>(*reinterpret_cast<const uint2*>(sd.codes + src), v);
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = u32(__floats2bfloat162_rn(v[2 * k] * s, v[2 * k + 1] * s));
        *reinterpret_cast<uint4*>((side ? V : K) + dst) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

template <int TYPE>
sb_status append_launch(sb_ctx* ctx, const Kv8Geom& g, const KvSide& ks, const KvSide& vs) {
    const int64_t maxb = ((int64_t)g.max_new + SB_KV8_BLOCK - 2) / SB_KV8_BLOCK + 1;     // blocks a request's new tokens can touch
    const int64_t units = maxb * g.heads * 2;
    if (units >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 append: max_new x heads too large");
    const dim3 grid((unsigned)((units + KA_WARPS - 1) / KA_WARPS), (unsigned)g.requests);
    if (g.dim <= 64) kv8_append_kernel<TYPE, 4><<<grid, KA_WARPS * 32, 0, ctx->stream>>>(g, ks, vs, ctx->dstate);
    else if (g.dim <= 128) kv8_append_kernel<TYPE, 8><<<grid, KA_WARPS * 32, 0, ctx->stream>>>(g, ks, vs, ctx->dstate);
    else kv8_append_kernel<TYPE, 16><<<grid, KA_WARPS * 32, 0, ctx->stream>>>(g, ks, vs, ctx->dstate);
    SB_LAUNCHED(ctx);
    return SB_OK;
}

}  // namespace

extern "C" sb_status sb_kv8_append(sb_ctx* ctx, const sb_kv8_cache* cache, const void* K, int64_t k_token_stride,
                                   int64_t k_head_stride, const void* V, int64_t v_token_stride, int64_t v_head_stride,
                                   int64_t total, const int32_t* starts, const int32_t* lens, int64_t max_new) {
    if (!ctx) return SB_ERR_INVALID;
    sb_status s = kv8_check(ctx, "kv8 append", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!K || !V) return sb_fail(ctx, SB_ERR_INVALID, "kv8 append: null");
    if (!kv8_aligned16(K) || !kv8_aligned16(V) || k_token_stride % 8 || k_head_stride % 8 || v_token_stride % 8 || v_head_stride % 8)
        return sb_fail(ctx, SB_ERR_SHAPE, "kv8 append: strides that are multiples of 8 and 16-byte aligned bases");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    const Kv8Geom g = kv8_geom(cache, total, starts, lens, max_new);
    const KvSide ks{static_cast<uint8_t*>(cache->k), static_cast<uint16_t*>(cache->k_scale),
                    static_cast<const __nv_bfloat16*>(K), k_token_stride, k_head_stride};
    const KvSide vs{static_cast<uint8_t*>(cache->v), static_cast<uint16_t*>(cache->v_scale),
                    static_cast<const __nv_bfloat16*>(V), v_token_stride, v_head_stride};
    return cache->type == SB_KV_INT8 ? append_launch<SB_KV_INT8>(ctx, g, ks, vs) : append_launch<SB_KV_E4M3>(ctx, g, ks, vs);
}

extern "C" sb_status sb_kv8_read(sb_ctx* ctx, const sb_kv8_cache* cache, int64_t total, const int32_t* starts,
                                 const int32_t* lens, int64_t max_new, void* K, void* V) {
    if (!ctx) return SB_ERR_INVALID;
    sb_status s = kv8_check(ctx, "kv8 read", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!K || !V) return sb_fail(ctx, SB_ERR_INVALID, "kv8 read: null");
    if (!kv8_aligned16(K) || !kv8_aligned16(V)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 read: 16-byte aligned outputs");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    const Kv8Geom g = kv8_geom(cache, total, starts, lens, max_new);
    const KvSide ks{static_cast<uint8_t*>(cache->k), static_cast<uint16_t*>(cache->k_scale), nullptr, 0, 0};
    const KvSide vs{static_cast<uint8_t*>(cache->v), static_cast<uint16_t*>(cache->v_scale), nullptr, 0, 0};
    const int64_t blocks = (max_new * g.heads * (g.dim / 8) + 255) / 256;
    if (blocks >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 read: max_new x heads too large");
    const dim3 grid((unsigned)blocks, (unsigned)g.requests);
    auto *k = static_cast<__nv_bfloat16*>(K), *v = static_cast<__nv_bfloat16*>(V);
    if (cache->type == SB_KV_INT8) kv8_read_kernel<SB_KV_INT8><<<grid, 256, 0, ctx->stream>>>(g, ks, vs, k, v, ctx->dstate);
    else kv8_read_kernel<SB_KV_E4M3><<<grid, 256, 0, ctx->stream>>>(g, ks, vs, k, v, ctx->dstate);
    SB_LAUNCHED(ctx);
    return SB_OK;
}
