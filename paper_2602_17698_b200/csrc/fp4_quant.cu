// Quantisation to the microscaled 4-bit formats and back.
//
// One thread takes 16 consecutive columns of a row: one 32-byte load (two of 16 bytes where rows are
// aligned no better), eight bytes of codes. That
// is one block of SB_FP4_NV; two neighbouring lanes share a block of SB_FP4_MX and exchange their
// maxima. The scales of four consecutive blocks are four consecutive bytes of a scale tile: the
// lanes that hold them pass them to the first, which stores one word. Nothing is read twice; the
// kernels move 2 + 1/2 + 1/16 (1/32) bytes an element. 14336 x 4096 there and back in MX: 51 to 53 us, 5.7 TB/s,
// 0.87 of a plain copy's rate, with 70 % of the issue slots used. NV to codes needs 16 instructions an element (an exact
// quotient, one number at a time) and is bound by their issue: 8192 x 4096 25 us, 77 % of the slots, where the bytes take 13.
#include "fp4.cuh"

namespace {

constexpr int FQ_THREADS = 256;
// Pieces of 16 columns a thread takes. With four the loads of a thread overlap and a block lives long
// enough to hide its start; a call with too few pieces for that takes one.
constexpr int FQ_MANY = 4;

// A row's pieces are counted through the whole matrix; index / pieces by a multiplication: with
// M = floor(2^64 / pieces) + 1, exact for index < 2^37 (checked) and pieces < 2^27.
struct FqDiv {
    uint64_t m;
    unsigned n;
    explicit FqDiv(int pieces) : m(pieces > 1 ? ~0ull / (unsigned)pieces + 1 : 0), n((unsigned)pieces) {}
#ifdef __CUDACC__
    __device__ __forceinline__ int64_t row(int64_t i, int& rest) const {
        const int64_t r = n > 1 ? (int64_t)__umul64hi((unsigned long long)i, m) : i;
        rest = (int)(i - r * n);
        return r;
    }
#endif
};

// 16 columns of a row as bf16 pairs; columns from `left` on read as zero
__device__ __forceinline__ void fq_load(const __nv_bfloat16* p, int64_t left, int wide, uint32_t (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0;
    if (left >= 16) {
        if (wide) ld_stream32(p, w);
        else {
            const uint4 a = ld_stream16(p), b = ld_stream16(p + 8);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
            w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        }
    } else if (left > 0) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < left) w[i >> 1] |= (uint32_t)q[i] << (16 * (i & 1));
    }
}
// codes of 16 columns and the scale byte of their block; g, rg: tensor scale and RN(1 / g)
template <int FORMAT>
__device__ __forceinline__ uint2 fq_codes(uint32_t (&w)[8], float g, float rg, uint32_t& scale) {
    // the largest magnitude as bf16 bits, whose order is the order of the numbers; a NaN stays one, above infinity
    __nv_bfloat162 m2 = __habs2(b162(w[0]));
#pragma unroll
    for (int i = 1; i < 8; ++i) m2 = __hmax2_nan(m2, __habs2(b162(w[i])));
    const uint32_t m = u32(m2);
    uint32_t amax = max(m & 0xffffu, m >> 16);
    float v[2][8];
    if (FORMAT == SB_FP4_MX) {
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        // floor(log2 amax) is the exponent of amax; below the smallest normal number the clamp decides
        const int e = (int)(amax >> 7) - 2;
        scale = amax >= 0x7f80u ? 255u : (uint32_t)max(e, 0);
        const float inv = __uint_as_float((254u - min(scale, 253u)) << 23);     // 2^-e, exact
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i >> 2][2 * (i & 3)] = bf16lo(w[i]) * inv;
            v[i >> 2][2 * (i & 3) + 1] = bf16hi(w[i]) * inv;
        }
    } else {
        const float am = __uint_as_float(amax << 16);
        // the two quotients the short way where everything stays in range
        const bool near = g > 0x1p-50f && g < 0x1p30f && am > 0x1p-60f && am < 0x1p60f;
        const float t = near ? div_rn(div_rn(am, 6.f, 0.16666667f), g, rg) : __fdiv_rn(__fdiv_rn(am, 6.f), g);
        // a quotient beyond the end of fp32 is one beyond the end of e4m3
        scale = amax >= 0x7f80u || !(g > 0.f) || !(t >= 0.f) ? 0x7fu : e4m3_of(fminf(t, 448.f));
        const float d = scale == 0x7fu ? 0.f : e4m3_value(scale) * g;
        if ((div_in_range(d) && t < 0x1p100f) || d == 0.f) {
            // x / d is at most 7 t / 448 where t passes 448, so it stays in range too; d = 0: every code is 0
            const float dd = d > 0.f ? d : 1.f, r1 = __frcp_rn(dd);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t x = d > 0.f ? w[i] : 0u;
                v[i >> 2][2 * (i & 3)] = div_rn(bf16lo(x), dd, r1);
                v[i >> 2][2 * (i & 3) + 1] = div_rn(bf16hi(x), dd, r1);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i >> 3][i & 7] = __fdiv_rn((i & 1) ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]), d);
        }
    }
    return make_uint2(fp4_pack8(v[0]), fp4_pack8(v[1]));
}

template <int FORMAT, int U>
__global__ void __launch_bounds__(FQ_THREADS)
fp4_quantize_kernel(const __nv_bfloat16* __restrict__ X, int64_t R, int64_t C, int64_t ldx, int64_t rows_padded,
                    const FqDiv div, int wide, const float* __restrict__ tensor_scale, uint8_t* __restrict__ codes,
                    uint8_t* __restrict__ scales) {
    const int64_t Cp = fp4_padded_cols(C);
    const float g = FORMAT == SB_FP4_NV && tensor_scale ? __ldg(tensor_scale) : 1.f, rg = __frcp_rn(g);
    const int64_t first = (int64_t)blockIdx.x * (FQ_THREADS * U) + threadIdx.x;
    uint32_t w[U][8];
    int64_t row[U];
    int piece[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        row[u] = div.row(first + u * FQ_THREADS, piece[u]);
        fq_load(X + row[u] * ldx + piece[u] * 16, row[u] < R ? C - (int64_t)piece[u] * 16 : 0, wide, w[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t scale;
        const uint2 q = fq_codes<FORMAT>(w[u], g, rg, scale);
        const int64_t r = row[u];
        const int64_t c0 = (int64_t)piece[u] * 16;
        const bool there = r < R && c0 < Cp;
        if (there) *reinterpret_cast<uint2*>(codes + r * (Cp >> 1) + (c0 >> 1)) = q;
        else scale = 0;                                        // padding rows and blocks
        constexpr int STEP = FORMAT == SB_FP4_MX ? 2 : 1;      // lanes per block
        uint32_t word = scale;
        word |= __shfl_down_sync(0xffffffffu, scale, STEP) << 8;
        word |= __shfl_down_sync(0xffffffffu, word, 2 * STEP) << 16;
        if (r < rows_padded && (piece[u] & (4 * STEP - 1)) == 0)
            *reinterpret_cast<uint32_t*>(scales + fp4_scale_at(r, piece[u] / STEP, div.n / (4 * STEP))) = word;
    }
}

// LOOSE: rows of Y are aligned to 2 or 4 bytes only.
template <int FORMAT, int U, bool LOOSE>
__global__ void __launch_bounds__(FQ_THREADS)
fp4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t R, int64_t C,
                      const FqDiv div, int64_t tiles, const float* __restrict__ tensor_scale, __nv_bfloat16* __restrict__ Y,
                      int64_t ldy, int align) {
    const float g = FORMAT == SB_FP4_NV && tensor_scale ? __ldg(tensor_scale) : 1.f;
    const int64_t first = (int64_t)blockIdx.x * (FQ_THREADS * U) + threadIdx.x;
    uint2 q[U];
    uint32_t s[U];
    int64_t row[U];
    int piece[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        row[u] = div.row(first + u * FQ_THREADS, piece[u]);
        if (row[u] < R) {
            q[u] = ld_stream8(codes + row[u] * (fp4_padded_cols(C) >> 1) + piece[u] * 8);
            s[u] = scales[fp4_scale_at(row[u], FORMAT == SB_FP4_MX ? piece[u] >> 1 : piece[u], tiles)];
        }
    }
    __shared__ uint4 words[LOOSE ? FQ_THREADS / 32 : 1][2 * 32];
    const int lane = threadIdx.x & 31;
    uint4* const mine = words[LOOSE ? threadIdx.x >> 5 : 0];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!LOOSE && row[u] >= R) break;
        const bool in = !LOOSE || row[u] < R;
        uint32_t o[8] = {};
        if (in) {
            const float d = FORMAT == SB_FP4_MX ? e8m0_value(s[u]) : e4m3_value(s[u]) * g;
            uint32_t h[2][4];
            fp4_unpack8(q[u].x, h[0]);
            fp4_unpack8(q[u].y, h[1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i >> 2][i & 3]));
                o[i] = u32(__floats2bfloat162_rn(f.x * d, f.y * d));
            }
        }
        const int64_t c0 = (int64_t)piece[u] * 16, at = row[u] * ldy + c0;
        if (!LOOSE && align == 32 && c0 + 16 <= C) {
            st_global32(Y + at, o);
            continue;
        }
        const int left = in ? (int)(C - c0 < 16 ? (C > c0 ? C - c0 : 0) : 16) : 0;
        if (!LOOSE) {
            if (left == 16) {
                *reinterpret_cast<uint4*>(Y + at) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(Y + at + 8) = make_uint4(o[4], o[5], o[6], o[7]);
            } else {
                uint16_t* p = reinterpret_cast<uint16_t*>(Y + at);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (i < left) p[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
            }
            continue;
        }
        // Rows that are aligned no better than their elements: the warp's 512 values change lanes, so that
        // a store of 32 lanes covers 128 consecutive bytes: 14336 x 4090 there and back (MX) 75 us, 365 with every lane
        // storing its own 16 values one by one.
        mine[2 * lane] = make_uint4(o[0], o[1], o[2], o[3]);
        mine[2 * lane + 1] = make_uint4(o[4], o[5], o[6], o[7]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int from = 4 * i + (lane >> 3), k = 2 * (lane & 7);
            const int64_t to = __shfl_sync(0xffffffffu, (long long)at, from) + k;
            const int there = __shfl_sync(0xffffffffu, left, from) - k;
            const uint32_t w = reinterpret_cast<const uint32_t*>(mine)[32 * i + lane];
            uint16_t* p = reinterpret_cast<uint16_t*>(Y + to);
            if (align >= 4 && there >= 2) *reinterpret_cast<uint32_t*>(p) = w;
            else {
                if (there >= 1) p[0] = (uint16_t)w;
                if (there >= 2) p[1] = (uint16_t)(w >> 16);
            }
        }
        __syncwarp();
    }
}

bool format_ok(int format) { return format == SB_FP4_MX || format == SB_FP4_NV; }
// four pieces a thread when that still makes 16 blocks per SM: quantising and restoring 14336 x 4096 in
// MX takes 51.3 us with four pieces and 53.4 with one, 28672 x 4096 96.8 and 101.5, but 4096 x 4096 20.5 and 18.6
bool fq_many(const sb_ctx* ctx, int64_t total) { return total >= (int64_t)FQ_THREADS * FQ_MANY * 16 * ctx->sm_count; }
unsigned fq_blocks(int64_t total, bool many) {
    const int64_t per = FQ_THREADS * (many ? FQ_MANY : 1);
    return (unsigned)((total + per - 1) / per);
}
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
    const FqDiv div((int)(fp4_scale_tiles(C, format) * 4 * fp4_block(format) / 16));
    const int64_t total = rows * div.n;
    if (total >= (1ll << 37)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 quantize: too many elements");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    auto* x = static_cast<const __nv_bfloat16*>(X);
    const int wide = ldx % 16 == 0 && (reinterpret_cast<uintptr_t>(X) & 31) == 0;
    const bool many = fq_many(ctx, total);
    const unsigned blocks = fq_blocks(total, many);
    auto launch = [&](auto kernel) { kernel<<<blocks, FQ_THREADS, 0, ctx->stream>>>(x, R, C, ldx, rows, div, wide, tensor_scale, codes, scales); };
    if (format == SB_FP4_MX) many ? launch(fp4_quantize_kernel<SB_FP4_MX, FQ_MANY>) : launch(fp4_quantize_kernel<SB_FP4_MX, 1>);
    else many ? launch(fp4_quantize_kernel<SB_FP4_NV, FQ_MANY>) : launch(fp4_quantize_kernel<SB_FP4_NV, 1>);
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
    const FqDiv div((int)((C + 15) / 16));
    const int64_t total = R * div.n, tiles = fp4_scale_tiles(C, format);
    if (total >= (1ll << 37)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 dequantize: too many elements");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    auto* y = static_cast<__nv_bfloat16*>(Y);
    const uintptr_t bits = reinterpret_cast<uintptr_t>(Y) | (uintptr_t)(2 * ldy);       // what every row is aligned to
    const int align = bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
    const bool many = fq_many(ctx, total);
    const unsigned blocks = fq_blocks(total, many);
    auto launch = [&](auto kernel) { kernel<<<blocks, FQ_THREADS, 0, ctx->stream>>>(codes, scales, R, C, div, tiles, tensor_scale, y, ldy, align); };
    auto by_size = [&](auto one, auto four) { many ? launch(four) : launch(one); };
    if (format == SB_FP4_MX) {
        if (align >= 16) by_size(fp4_dequantize_kernel<SB_FP4_MX, 1, false>, fp4_dequantize_kernel<SB_FP4_MX, FQ_MANY, false>);
        else by_size(fp4_dequantize_kernel<SB_FP4_MX, 1, true>, fp4_dequantize_kernel<SB_FP4_MX, FQ_MANY, true>);
    } else {
        if (align >= 16) by_size(fp4_dequantize_kernel<SB_FP4_NV, 1, false>, fp4_dequantize_kernel<SB_FP4_NV, FQ_MANY, false>);
        else by_size(fp4_dequantize_kernel<SB_FP4_NV, 1, true>, fp4_dequantize_kernel<SB_FP4_NV, FQ_MANY, true>);
    }
    SB_LAUNCHED(ctx);
    return SB_OK;
}
