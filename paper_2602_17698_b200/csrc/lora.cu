// What low-rank adapters add to a shared projection: Y = base + scale B (A x), the adapter by request.
//
// Two kernels: the first leaves H = A x (fp32, rank numbers a row) in scratch, split along `in` where rows are few, the second adds
// the splits' sums, multiplies with B and adds the base. Both products run on mma.sync m16n8k16 with rows on the 16-row side: they
// are a few operations a byte, so the bytes of X, of base and Y and of the adapters bound them, and tcgen05 would have nothing to
// win. The contraction may visit its index in any order: a lane takes consecutive elements of its operand rows, so both operands go
// from global memory straight into registers, 16 bytes at a time. In the second product a lane's columns are made consecutive
// too (column 8 (n / 2) + 2 j + n % 2 is column n of tile j), so base and Y move in 16-byte pieces.
//
// H is held for the second product as the sum of two bf16 numbers, h = hi + lo with lo = bf16(h - hi): what is lost is
// below 2^-17 of h, so the result's one rounding decides.
#include "kv8.cuh"

namespace {

struct LoArgs {
    const __nv_bfloat16 *x, *a, *b;
    const float* scale;
    const void* base;
    void* y;
    int64_t ldx, ld_base, ldy, in, out, total;
    const int32_t *starts, *ids;
    int requests, adapters, rank, max_new;
    int direct;                  // a row tile per request (no request has more rows), else tiles of all requests one after the other
    int splits;                  // of `in`
    int64_t columns;             // of a block of the second kernel, a multiple of 32
    float* h;                    // [splits][total][padded rank]
    SbDeviceState* st;
};

__device__ __forceinline__ void lo_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lo_ld16(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

struct LoTile { int64_t row0; int rows, adapter; };
// The rows of a request; none (and the status latched) where its numbers do not fit.
__device__ __forceinline__ int lo_rows(const LoArgs& a, int b, int64_t& row0) {
    row0 = a.starts[b];
    const int64_t n = (int64_t)a.starts[b + 1] - row0;
    if (row0 >= 0 && n >= 0 && n <= a.max_new && row0 + n <= a.total) return (int)n;
    sb_latch(a.st, SB_ERR_INVALID, SBK_LORA);
    return 0;
}
// Tile number `tile`; all threads of the block take part. rows = 0: there is no such tile.
template <int TM, int THREADS>
__device__ __forceinline__ LoTile lo_tile(const LoArgs& a, int tile) {
    LoTile t{0, 0, -1};
    int b = tile;
    int64_t row0;
    if (a.direct) {
        t.rows = lo_rows(a, b, row0);
        t.row0 = row0;
    } else {
        __shared__ int sums[THREADS / 32], found[2];
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (threadIdx.x == 0) found[0] = -1;
        int before = 0;
        for (int base = 0; base < a.requests; base += THREADS) {
            const int r = base + threadIdx.x;
            const int mine = r < a.requests ? (lo_rows(a, r, row0) + TM - 1) / TM : 0;
            int x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            __syncthreads();
            if (lane == 31) sums[warp] = x;
            __syncthreads();
            int all = 0, below = before;
#pragma unroll
            for (int w = 0; w < THREADS / 32; ++w) {
                if (w < warp) below += sums[w];
                all += sums[w];
            }
            const int lo = below + x - mine;
            if (tile >= lo && tile < lo + mine) {
                found[0] = r;
                found[1] = tile - lo;
            }
            before += all;
            if (tile < before) break;
        }
        __syncthreads();
        b = found[0];
        if (b < 0) return t;
        const int n = lo_rows(a, b, row0);
        t.row0 = row0 + (int64_t)found[1] * TM;
        t.rows = min(TM, n - found[1] * TM);
    }
    t.adapter = a.ids[b];
    if (t.adapter < -1 || t.adapter >= a.adapters) {
        sb_latch(a.st, SB_ERR_INVALID, SBK_LORA);
        t.adapter = -1;
    }
    return t;
}

// ---- H = A x ----
// 8 warps: MG groups of 16 rows, 8 / MG parts of the block's range of `in`.
template <int RP, int MG>
__global__ void __launch_bounds__(256)
lora_down_kernel(const LoArgs a) {
    constexpr int KG = 8 / MG, NT = RP / 8, TM = 16 * MG;
    extern __shared__ __align__(16) float lo_sums[];                 // [KG][TM][RP]
    const LoTile tile = lo_tile<TM, 256>(a, blockIdx.x);
    if (tile.rows <= 0 || tile.adapter < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int mg = warp % MG, kg = warp / MG;
    const int64_t units = (a.in + 31) / 32, parts = (int64_t)a.splits * KG, part = (int64_t)blockIdx.y * KG + kg;
    const int64_t u0 = units * part / parts, u1 = units * (part + 1) / parts;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
    const int r0 = 16 * mg + g, r1 = r0 + 8;
    const __nv_bfloat16 *x0 = a.x + (tile.row0 + min(r0, tile.rows - 1)) * a.ldx + 8 * t, *x1 = a.x + (tile.row0 + min(r1, tile.rows - 1)) * a.ldx + 8 * t;
    const __nv_bfloat16* w = a.a + ((int64_t)tile.adapter * a.rank + g) * a.in + 8 * t;
    const bool live = 16 * mg < tile.rows;
#pragma unroll 2
    for (int64_t u = u0; live && u < u1; ++u) {
        const int64_t k = 32 * u;
        const bool in = k + 8 * t < a.in;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const uint4 p = in && r0 < tile.rows ? lo_ld16(x0 + k) : zero, q = in && r1 < tile.rows ? lo_ld16(x1 + k) : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint4 v = in && 8 * n < a.rank ? lo_ld16(w + 8 * n * a.in + k) : zero;
            lo_mma(acc[n], p.x, q.x, p.y, q.y, v.x, v.y);
            lo_mma(acc[n], p.z, q.z, p.w, q.w, v.z, v.w);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* s = lo_sums + ((kg * TM + r0) * RP + 8 * n + 2 * t);
        *reinterpret_cast<float2*>(s) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(s + 8 * RP) = make_float2(acc[n][2], acc[n][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tile.rows * RP; i += 256) {
        float sum = lo_sums[i];
#pragma unroll
        for (int k = 1; k < KG; ++k) sum += lo_sums[k * TM * RP + i];
        a.h[((int64_t)blockIdx.y * a.total + tile.row0) * RP + i] = sum;
    }
}

// ---- Y = base + scale B H ----
template <typename T> struct LoOut;
template <> struct LoOut<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, bool wide) {
        if (wide && left >= 8) v = *reinterpret_cast<const uint4*>(p);
        else {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) w[i >> 1] |= (uint32_t)q[i] << (16 * (i & 1));
            v = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ __forceinline__ void add(const float (&x)[8], float f) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = u32(__floats2bfloat162_rn(fmaf(x[2 * i], f, bf16lo(w[i])), fmaf(x[2 * i + 1], f, bf16hi(w[i]))));
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p, int left, bool wide) const {
        if (wide && left >= 8) *reinterpret_cast<uint4*>(p) = v;
        else {
            uint16_t* q = reinterpret_cast<uint16_t*>(p);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) q[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
};
template <> struct LoOut<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* p, int left, bool wide) {
        if (wide && left >= 8) {
            const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
        }
    }
    __device__ __forceinline__ void add(const float (&x)[8], float f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(x[i], f, v[i]);
    }
    __device__ __forceinline__ void store(float* p, int left, bool wide) const {
        if (wide && left >= 8) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = v[i];
        }
    }
};

// 8 warps: RG groups of 16 MW rows, 8 / RG groups of 32 columns. RP: rank rounded up to 16, 32, 64 or 128.
template <int RP, int MW, int RG, typename T>
__global__ void __launch_bounds__(256)
lora_up_kernel(const LoArgs a, const int wide) {
    constexpr int TM = 16 * MW * RG, CG = 8 / RG, KS = RP / 16, KW = RP / 8;       // KW: words of a row that a lane takes
    const LoTile tile = lo_tile<TM, 256>(a, blockIdx.x);
    if (tile.rows <= 0) return;
    const T* base = static_cast<const T*>(a.base) + tile.row0 * a.ld_base;
    T* const y = static_cast<T*>(a.y) + tile.row0 * a.ldy;
    const int64_t c0 = (int64_t)blockIdx.y * a.columns, c1 = min(a.out, c0 + a.columns);
    if (tile.adapter < 0) {
        if (base != y) {
            for (int r = threadIdx.x >> 5; r < tile.rows; r += 8)
                for (int64_t c = c0 + 8 * (threadIdx.x & 31); c < c1; c += 256) {
                    LoOut<T> v;
                    const int left = (int)min((int64_t)8, c1 - c);
                    v.load(base + r * a.ld_base + c, left, wide);
                    v.store(y + r * a.ldy + c, left, wide);
                }
        }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rg = warp % RG, cg = warp / RG;
    if (16 * MW * rg >= tile.rows) return;
    const float scale = a.scale ? __ldg(a.scale + tile.adapter) : 1.f;
    const int kl = a.rank / 4;                                       // elements of a row of B that a lane takes, from kl t on
    // operands of H: word i of a lane is elements kl t + 2 i, + 1
    uint32_t hi[MW][2][KW], lo[MW][2][KW];
#pragma unroll
    for (int m = 0; m < MW; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 16 * (MW * rg + m) + g + 8 * e;
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                float2 v = make_float2(0.f, 0.f);
                if (r < tile.rows && 2 * i < kl) {
                    const float* h = a.h + (tile.row0 + r) * RP + kl * t + 2 * i;
                    v = *reinterpret_cast<const float2*>(h);
                    for (int s = 1; s < a.splits; ++s) {
                        const float2 w = *reinterpret_cast<const float2*>(h + (int64_t)s * a.total * RP);
                        v.x += w.x;
                        v.y += w.y;
                    }
                }
                const uint32_t top = u32(__floats2bfloat162_rn(v.x, v.y));
                hi[m][e][i] = top;
                // (of an infinity nothing is left)
                const float x = v.x - bf16lo(top), y = v.y - bf16hi(top);
                lo[m][e][i] = u32(__floats2bfloat162_rn(fabsf(bf16lo(top)) < INFINITY ? x : 0.f, fabsf(bf16hi(top)) < INFINITY ? y : 0.f));
            }
        }
    const __nv_bfloat16* w = a.b + (int64_t)tile.adapter * a.out * a.rank + kl * t;
    for (int64_t c = c0 + 32 * cg; c < c1; c += 32 * CG) {
        float acc[MW][4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // column n of tile j is c + 8 (n / 2) + 2 j + n % 2
            const int64_t col = c + 8 * (g >> 1) + 2 * j + (g & 1);
            uint32_t v[KW];
            const __nv_bfloat16* p = w + col * a.rank;
            if (col >= c1) {
#pragma unroll
                for (int i = 0; i < KW; ++i) v[i] = 0;
            } else if (a.rank == RP && RP >= 32) {
#pragma unroll
                for (int i = 0; i < KW / 4; ++i) {
                    const uint4 x = lo_ld16(p + 8 * i);
                    v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
                }
            } else if (a.rank == 16 && RP == 16) {
                const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
                v[0] = x.x; v[1] = x.y;
            } else {
#pragma unroll
                for (int i = 0; i < KW; ++i) v[i] = 2 * i < kl ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
            }
#pragma unroll
            for (int m = 0; m < MW; ++m) {
                acc[m][j][0] = acc[m][j][1] = acc[m][j][2] = acc[m][j][3] = 0.f;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    lo_mma(acc[m][j], lo[m][0][2 * s], lo[m][1][2 * s], lo[m][0][2 * s + 1], lo[m][1][2 * s + 1], v[2 * s], v[2 * s + 1]);
                    lo_mma(acc[m][j], hi[m][0][2 * s], hi[m][1][2 * s], hi[m][0][2 * s + 1], hi[m][1][2 * s + 1], v[2 * s], v[2 * s + 1]);
                }
            }
        }
        const int64_t col = c + 8 * t;                               // a lane's eight columns
        const int left = (int)min((int64_t)8, c1 - col);
        if (left <= 0) continue;
#pragma unroll
        for (int m = 0; m < MW; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 16 * (MW * rg + m) + g + 8 * e;
                if (r >= tile.rows) continue;
                const float x[8] = {acc[m][0][2 * e], acc[m][0][2 * e + 1], acc[m][1][2 * e], acc[m][1][2 * e + 1],
                                    acc[m][2][2 * e], acc[m][2][2 * e + 1], acc[m][3][2 * e], acc[m][3][2 * e + 1]};
                LoOut<T> o;
                o.load(base + r * a.ld_base + col, left, wide);
                o.add(x, scale);
                o.store(y + r * a.ldy + col, left, wide);
            }
    }
}

template <int RP, int MG>
sb_status down_launch(sb_ctx* ctx, const LoArgs& a, int64_t tiles) {
    auto* kernel = lora_down_kernel<RP, MG>;
    constexpr int smem = 8 * 16 * RP * 4;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    kernel<<<dim3((unsigned)tiles, (unsigned)a.splits), 256, smem, ctx->stream>>>(a);
    SB_LAUNCHED(ctx);
    return SB_OK;
}
template <int RP, int MW, int RG>
sb_status up_launch(sb_ctx* ctx, const LoArgs& a, int64_t tiles, int f32, int wide) {
    const dim3 grid((unsigned)tiles, (unsigned)((a.out + a.columns - 1) / a.columns));
    if (f32) lora_up_kernel<RP, MW, RG, float><<<grid, 256, 0, ctx->stream>>>(a, wide);
    else lora_up_kernel<RP, MW, RG, __nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(a, wide);
    SB_LAUNCHED(ctx);
    return SB_OK;
}

// Rows of a tile of either kernel: 16 where every request fits into that, else 64.
template <int RP>
sb_status lo_run(sb_ctx* ctx, LoArgs& a, int f32, int wide) {
    a.direct = a.max_new <= 16;
    const int64_t tiles = a.direct ? a.requests : (a.total + 63) / 64 + a.requests;
    if (tiles >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "lora: too many rows");
    // parts of `in`: four blocks a multiprocessor, of 1024 at least
    int64_t splits = 4 * ctx->sm_count / tiles, most = (a.in + 1023) / 1024;
    splits = splits > most ? most : splits;
    a.splits = splits < 1 ? 1 : (int)splits;
    void* arena;
    sb_status s = sb_scratch(ctx, Carver::need({(size_t)a.splits * (size_t)a.total * RP * 4}), &arena);
    if (s != SB_OK) return s;
    a.h = Carver(arena).take<float>((size_t)a.splits * (size_t)a.total * RP);
    // columns of a block of the second kernel: eight blocks a multiprocessor
    int64_t parts = 8 * ctx->sm_count / tiles, unit = a.direct ? 256 : 32 * (RP == 128 ? 2 : 4);
    most = (a.out + unit - 1) / unit;
    parts = parts > most ? most : parts;
    if (parts < 1) parts = 1;
    if (parts > 65535) parts = 65535;
    a.columns = (most + parts - 1) / parts * unit;
    if (a.direct) {
        s = down_launch<RP, 1>(ctx, a, tiles);
        return s != SB_OK ? s : up_launch<RP, 1, 1>(ctx, a, tiles, f32, wide);
    }
    s = down_launch<RP, 4>(ctx, a, tiles);
    if (s != SB_OK) return s;
    if constexpr (RP == 128) return up_launch<RP, 1, 4>(ctx, a, tiles, f32, wide);
    else return up_launch<RP, 2, 2>(ctx, a, tiles, f32, wide);
}

}  // namespace

extern "C" sb_status sb_lora_add(sb_ctx* ctx, const sb_lora_adapters* ad, const void* X, int64_t ldx, const void* base, int64_t ld_base,
                                 void* Y, int64_t ldy, int f32, int64_t total, const int32_t* starts, const int32_t* ids, int requests,
                                 int64_t max_new) {
    if (!ctx) return SB_ERR_INVALID;
    if (!ad || !ad->a || !ad->b || !starts || !ids) return sb_fail(ctx, SB_ERR_INVALID, "lora: null");
    if (ad->adapters < 1 || ad->in < 1 || ad->out < 1 || total < 0 || max_new < 0 || requests < 0 || (f32 != 0 && f32 != 1))
        return sb_fail(ctx, SB_ERR_INVALID, "lora: no adapters, or negative sizes");
    if (ad->rank < 8 || ad->rank > 128 || ad->rank % 8 || ad->in % 8) return sb_fail(ctx, SB_ERR_SHAPE, "lora: rank 8 to 128, rank and in multiples of 8");
    if (total == 0 || max_new == 0 || requests == 0) return SB_OK;
    if (!X || !base || !Y) return sb_fail(ctx, SB_ERR_INVALID, "lora: null");
    if (requests > 65535 || total >= (1ll << 31) || max_new >= (1ll << 31) || ad->in >= (1ll << 31) || ad->out >= (1ll << 31))
        return sb_fail(ctx, SB_ERR_SHAPE, "lora: at most 65535 requests and 2^31 rows and columns");
    const int size = f32 ? 4 : 2;
    const uintptr_t ends = reinterpret_cast<uintptr_t>(base) | reinterpret_cast<uintptr_t>(Y);
    if (total > 1 && (ldx < ad->in || ld_base < ad->out || ldy < ad->out)) return sb_fail(ctx, SB_ERR_SHAPE, "lora: rows longer than their leading dimension");
    if (!kv8_aligned16(X) || !kv8_aligned16(ad->a) || !kv8_aligned16(ad->b) || (total > 1 && ldx % 8) || (ends & (size - 1)))
        return sb_fail(ctx, SB_ERR_SHAPE, "lora: 16-byte aligned X, a and b, ldx a multiple of 8, base and Y aligned to their type");
    if (Y == base && total > 1 && ldy != ld_base) return sb_fail(ctx, SB_ERR_SHAPE, "lora: in place with another leading dimension");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    LoArgs a{};
    a.x = static_cast<const __nv_bfloat16*>(X); a.a = static_cast<const __nv_bfloat16*>(ad->a); a.b = static_cast<const __nv_bfloat16*>(ad->b);
    a.scale = ad->scale; a.base = base; a.y = Y;
    a.ldx = ldx; a.ld_base = ld_base; a.ldy = ldy; a.in = ad->in; a.out = ad->out; a.total = total;
    a.starts = starts; a.ids = ids; a.requests = requests; a.adapters = ad->adapters; a.rank = ad->rank;
    a.max_new = (int)max_new; a.st = ctx->dstate;
    const int wide = (ends & 15) == 0 && (total == 1 || ((ld_base * size) % 16 == 0 && (ldy * size) % 16 == 0));
    return ad->rank <= 16 ? lo_run<16>(ctx, a, f32, wide) : ad->rank <= 32 ? lo_run<32>(ctx, a, f32, wide)
         : ad->rank <= 64 ? lo_run<64>(ctx, a, f32, wide) : lo_run<128>(ctx, a, f32, wide);
}
