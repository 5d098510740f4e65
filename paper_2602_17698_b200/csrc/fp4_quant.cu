// Quantisation to the microscaled 4-bit formats and back.
//
// One thread takes 16 consecutive columns of a row: two 16-byte loads, eight bytes of codes. That
// is one block of SB_FP4_NV; two neighbouring lanes share a block of SB_FP4_MX and exchange their
// maxima. The scales of four consecutive blocks are four consecutive bytes of a scale tile: the
// lanes that hold them pass them to the first, which stores one word. Nothing is read twice; the
// kernels move 2 + 1/2 + 1/16 (1/32) bytes an element and are bound by that traffic.
#include "fp4.cuh"

namespace {

constexpr int FQ_THREADS = 256;

// x / d for every element of a block at the price of three instructions instead of a division:
// with r = RN(1 / d) and q = RN(x r), RN(q + r (x - q d)) is the correctly rounded quotient
// (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).
// It needs r, q and the residual in the range of normal numbers: d between 2^-100 and 2^100 (a
// quotient that underflows then is far below the smallest code and rounds to 0 either way).
__device__ __forceinline__ float quotient(float x, float d, float r, bool plain) {
    if (plain) return __fdiv_rn(x, d);
    const float q = x * r;
    return copysignf(fmaf(fmaf(-q, d, x), r, q), x);         // -0 would come out as 0
}

template <int FORMAT>
__global__ void __launch_bounds__(FQ_THREADS)
fp4_quantize_kernel(const __nv_bfloat16* __restrict__ X, int64_t R, int64_t C, int64_t ldx, int64_t rows_padded,
                    int units, const float* __restrict__ tensor_scale, uint8_t* __restrict__ codes,
                    uint8_t* __restrict__ scales) {
    // units: groups of 16 columns of a row, a whole number of scale tiles
    const int64_t first = (int64_t)blockIdx.x * FQ_THREADS;
    const int64_t row0 = first / units;
    const unsigned off = (unsigned)(first - row0 * units) + threadIdx.x;
    const int64_t r = row0 + off / (unsigned)units;
    const int u = (int)(off % (unsigned)units);
    const int64_t c0 = (int64_t)u * 16;
    const int64_t Cp = fp4_padded_cols(C);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0;
    if (r < R && c0 < C) {
        const __nv_bfloat16* p = X + r * ldx + c0;
        if (c0 + 16 <= C) {
            const uint4 a = ld_stream16(p), b = ld_stream16(p + 8);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
            w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        } else {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c0 + i < C) w[i >> 1] |= (uint32_t)q[i] << (16 * (i & 1));
        }
    }
    // the largest magnitude as bf16 bits: their order is the order of the numbers, NaN above infinity
    uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    uint32_t amax = max(m & 0xffffu, m >> 16);
    if (FORMAT == SB_FP4_MX) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));

    float v[16];
    uint32_t scale;
    if (FORMAT == SB_FP4_MX) {
        // floor(log2 amax) is the exponent of amax; below the smallest normal number the clamp decides
        const int e = (int)(amax >> 7) - 2;
        scale = amax >= 0x7f80u ? 255u : (uint32_t)max(e, 0);
        const float inv = __uint_as_float((254u - min(scale, 253u)) << 23);     // 2^-e, exact
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = bf16lo(w[i]) * inv;
            v[2 * i + 1] = bf16hi(w[i]) * inv;
        }
    } else {
        const float g = tensor_scale ? __ldg(tensor_scale) : 1.f;
        const float t = __fdiv_rn(__fdiv_rn(__uint_as_float(amax << 16), 6.f), g);
        scale = !(g > 0.f) || !(t >= 0.f && t < __uint_as_float(0x7f800000u)) ? 0x7fu : e4m3_of(t);
        const float d = scale == 0x7fu ? 0.f : e4m3_value(scale) * g;
        const bool plain = !(d > 0x1p-100f && d < 0x1p100f);
        const float r1 = __frcp_rn(d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = d > 0.f ? quotient(bf16lo(w[i]), d, r1, plain) : 0.f;
            v[2 * i + 1] = d > 0.f ? quotient(bf16hi(w[i]), d, r1, plain) : 0.f;
        }
    }
    if (r < R && c0 < Cp) {
        const float (&lo)[8] = *reinterpret_cast<float (*)[8]>(&v[0]);
        const float (&hi)[8] = *reinterpret_cast<float (*)[8]>(&v[8]);
        *reinterpret_cast<uint2*>(codes + r * (Cp >> 1) + (c0 >> 1)) = make_uint2(fp4_pack8(lo), fp4_pack8(hi));
    }
    // padding rows and blocks: 0
    if (r >= R || c0 >= Cp) scale = 0;
    constexpr int STEP = FORMAT == SB_FP4_MX ? 2 : 1;          // lanes per block
    uint32_t word = scale;
    word |= __shfl_down_sync(0xffffffffu, scale, STEP) << 8;
    word |= __shfl_down_sync(0xffffffffu, word, 2 * STEP) << 16;
    if (r < rows_padded && (u & (4 * STEP - 1)) == 0)
        *reinterpret_cast<uint32_t*>(scales + fp4_scale_at(r, u / STEP, units / (4 * STEP))) = word;
}

template <int FORMAT>
__global__ void __launch_bounds__(FQ_THREADS)
fp4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t R, int64_t C,
                      int units, int64_t tiles, const float* __restrict__ tensor_scale, __nv_bfloat16* __restrict__ Y,
                      int64_t ldy, int wide) {
    const int64_t first = (int64_t)blockIdx.x * FQ_THREADS;
    const int64_t row0 = first / units;
    const unsigned off = (unsigned)(first - row0 * units) + threadIdx.x;
    const int64_t r = row0 + off / (unsigned)units;
    const int u = (int)(off % (unsigned)units);
    if (r >= R) return;
    const int64_t c0 = (int64_t)u * 16;
    const uint2 q = *reinterpret_cast<const uint2*>(codes + r * (fp4_padded_cols(C) >> 1) + (c0 >> 1));
    const uint32_t s = scales[fp4_scale_at(r, FORMAT == SB_FP4_MX ? u >> 1 : u, tiles)];
    float d;
    if (FORMAT == SB_FP4_MX) d = e8m0_value(s);
    else d = e4m3_value(s) * (tensor_scale ? __ldg(tensor_scale) : 1.f);
    uint32_t h[8];
    fp4_unpack8(q.x, *reinterpret_cast<uint32_t (*)[4]>(&h[0]));
    fp4_unpack8(q.y, *reinterpret_cast<uint32_t (*)[4]>(&h[4]));
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        o[i] = u32(__floats2bfloat162_rn(f.x * d, f.y * d));
    }
    __nv_bfloat16* y = Y + r * ldy + c0;
    if (wide && c0 + 16 <= C) {
        reinterpret_cast<uint4*>(y)[0] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4*>(y)[1] = make_uint4(o[4], o[5], o[6], o[7]);
    } else {
        uint16_t* p = reinterpret_cast<uint16_t*>(y);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c0 + i < C) p[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
    }
}

bool format_ok(int format) { return format == SB_FP4_MX || format == SB_FP4_NV; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

extern "C" int64_t sb_fp4_code_bytes(int64_t R, int64_t C) {
    if (R <= 0 || C <= 0) return -1;
    return R * (fp4_padded_cols(C) / 2);
}
extern "C" int64_t sb_fp4_scale_bytes(int64_t R, int64_t C, int format) {
    if (R <= 0 || C <= 0 || !format_ok(format)) return -1;
    return ((R + 127) / 128) * fp4_scale_tiles(C, format) * 512;
}

extern "C" sb_status sb_fp4_quantize(sb_ctx* ctx, const void* X, int64_t R, int64_t C, int64_t ldx, int format,
                                     const float* tensor_scale, uint8_t* codes, uint8_t* scales) {
    if (!ctx) return SB_ERR_INVALID;
    if (!X || !codes || !scales || R <= 0 || C <= 0) return sb_fail(ctx, SB_ERR_INVALID, "fp4 quantize: null or empty");
    if (!format_ok(format)) return sb_fail(ctx, SB_ERR_INVALID, "fp4 quantize: unknown format %d", format);
    if (format == SB_FP4_MX && tensor_scale)
        return sb_fail(ctx, SB_ERR_INVALID, "fp4 quantize: SB_FP4_MX has no tensor scale");
    if (ldx % 8 || ldx < C || !aligned16(X) || !aligned16(codes) || !aligned16(scales))
        return sb_fail(ctx, SB_ERR_SHAPE, "fp4 quantize: ldx %% 8 == 0, ldx >= C and 16-byte aligned pointers");
    if (R >= (1ll << 31) - 128 || C >= (1ll << 30)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 quantize: R and C must fit 31 bits");
    const int64_t rows = (R + 127) / 128 * 128;
    const int units = (int)(fp4_scale_tiles(C, format) * 4 * fp4_block(format) / 16);
    const int64_t blocks = (rows * units + FQ_THREADS - 1) / FQ_THREADS;
    if (blocks >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 quantize: too many elements");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    auto* x = static_cast<const __nv_bfloat16*>(X);
    if (format == SB_FP4_MX)
        fp4_quantize_kernel<SB_FP4_MX><<<(unsigned)blocks, FQ_THREADS, 0, ctx->stream>>>(x, R, C, ldx, rows, units, nullptr, codes, scales);
    else
        fp4_quantize_kernel<SB_FP4_NV><<<(unsigned)blocks, FQ_THREADS, 0, ctx->stream>>>(x, R, C, ldx, rows, units, tensor_scale, codes, scales);
    SB_LAUNCHED(ctx);
    return SB_OK;
}

extern "C" sb_status sb_fp4_dequantize(sb_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t R, int64_t C,
                                       int format, const float* tensor_scale, void* Y, int64_t ldy) {
    if (!ctx) return SB_ERR_INVALID;
    if (!Y || !codes || !scales || R <= 0 || C <= 0) return sb_fail(ctx, SB_ERR_INVALID, "fp4 dequantize: null or empty");
    if (!format_ok(format)) return sb_fail(ctx, SB_ERR_INVALID, "fp4 dequantize: unknown format %d", format);
    if (format == SB_FP4_MX && tensor_scale)
        return sb_fail(ctx, SB_ERR_INVALID, "fp4 dequantize: SB_FP4_MX has no tensor scale");
    if (ldy < C || !aligned16(codes) || !aligned16(scales) || (reinterpret_cast<uintptr_t>(Y) & 1))
        return sb_fail(ctx, SB_ERR_SHAPE, "fp4 dequantize: ldy >= C and 16-byte aligned codes and scales");
    if (R >= (1ll << 31) - 128 || C >= (1ll << 30)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 dequantize: R and C must fit 31 bits");
    const int units = (int)((C + 15) / 16);
    const int64_t blocks = (R * units + FQ_THREADS - 1) / FQ_THREADS;
    if (blocks >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 dequantize: too many elements");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    auto* y = static_cast<__nv_bfloat16*>(Y);
    const int wide = ldy % 8 == 0 && aligned16(Y);
    const int64_t tiles = fp4_scale_tiles(C, format);
    if (format == SB_FP4_MX)
        fp4_dequantize_kernel<SB_FP4_MX><<<(unsigned)blocks, FQ_THREADS, 0, ctx->stream>>>(codes, scales, R, C, units, tiles, nullptr, y, ldy, wide);
    else
        fp4_dequantize_kernel<SB_FP4_NV><<<(unsigned)blocks, FQ_THREADS, 0, ctx->stream>>>(codes, scales, R, C, units, tiles, tensor_scale, y, ldy, wide);
    SB_LAUNCHED(ctx);
    return SB_OK;
}
