// Products of microscaled 4-bit matrices on the block-scaled tensor core instructions
// (tcgen05.mma kind::mxf4 / kind::mxf4nvf4): Y[m][n] = gA gB sum_k A[m][k] B[n][k].
//
// The rows of B (weights) lie on the instruction's 128-row side and the rows of A (tokens) on its
// other side, so that a decode batch fills an instruction whatever its size: the accumulator holds
// Y transposed, lane = weight row, column = token, and 32 lanes store 32 consecutive outputs of a
// token. Codes come by TMA (128-byte swizzle, 256 columns a row), scales by one contiguous copy per
// operand (a slab's scale tiles are neighbours in memory), and go from shared to tensor memory by
// tcgen05.cp, which spreads a scale tile's 32 x 16 bytes over the lanes as the instruction reads
// them. No thread touches a code.
//
// fp4_tile_kernel: one CTA per 128 weight rows x NT tokens; with few tiles the columns are cut into
// segments, the CTAs of a cluster, added in segment order through distributed shared memory.
#include <cooperative_groups.h>

#include "fp4.cuh"
#include "tensor5.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int FG_ROWS = 128;             // weight rows of a tile
constexpr int FG_SLAB = 256;             // columns per ring stage: 128 bytes of codes
constexpr int FG_MAX_SPLIT = 8;          // portable cluster size
constexpr int FG_THREADS = 192;          // warp 0: copies, warp 1: products, warps 2-5: results

struct FgArgs {
    const uint8_t* w_scales;             // [row tiles][tiles][512]
    const uint8_t* x_scales;
    int64_t tiles;                       // scale tiles along K
    const float *w_tensor, *x_tensor;    // or NULL
    int64_t M, N;                        // tokens, weight rows
    int slabs, k64;                      // ring stages and instruction steps along K
    void* Y;
    int64_t ldy;
    int out_f32;
    SbDeviceState* st;
};

template <int FORMAT, int NT>
struct FgShape {
    static constexpr int ATOMS = FORMAT == SB_FP4_MX ? 2 : 4;        // scale tiles of a slab
    static constexpr int W_BYTES = FG_ROWS * 128, X_BYTES = NT * 128, S_BYTES = ATOMS * 512;
    static constexpr int STAGE = W_BYTES + X_BYTES + 2 * S_BYTES;
    static constexpr int STAGES = 4;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 256;
    static constexpr int SF_COLS = 2 * 4 * ATOMS;                    // scale columns of a stage
    static constexpr int D_COLS = NT < 32 ? 32 : NT;
    static constexpr int TMEM = D_COLS + STAGES * SF_COLS <= 128 ? 128 : 256;
    static_assert(D_COLS + STAGES * SF_COLS <= 256, "tensor memory of two CTAs of an SM");
    static_assert(FG_ROWS * NT * 4 <= STAGES * STAGE, "partial sums fit where the ring was");
};

// Instruction descriptor: e2m1 x e2m1, both K-major, M = m, N = n, the scale format, and which half
// of a 32-bit scale cell the step reads (MX keeps two steps' scales in a cell).
template <int FORMAT>
__device__ __forceinline__ constexpr unsigned fg_idesc(int m, int n, int half) {
    return 1u << 7 | 1u << 10 | (unsigned)(n >> 3) << 17 | (FORMAT == SB_FP4_MX ? 1u << 23 : 0u) | (unsigned)(m >> 7) << 27 |
           (unsigned)(2 * half) << 4 | (unsigned)(2 * half) << 29;
}
template <int FORMAT>
__device__ __forceinline__ void fg_mma(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sa,
                                       unsigned sb, unsigned accumulate) {
    if (FORMAT == SB_FP4_MX)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void fg_copy_scales(unsigned taddr, unsigned smem) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(t5_desc_rows16(smem)) : "memory");
}
__device__ __forceinline__ void fg_commit(unsigned bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fg_store(const FgArgs& a, int64_t m, int64_t n, float v) {
    if (a.out_f32) static_cast<float*>(a.Y)[m * a.ldy + n] = v;
    else static_cast<__nv_bfloat16*>(a.Y)[m * a.ldy + n] = __float2bfloat16_rn(v);
}

template <int FORMAT, int NT>
__global__ void __launch_bounds__(FG_THREADS)
fp4_tile_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const FgArgs a) {
    using S = FgShape<FORMAT, NT>;
    extern __shared__ unsigned char fg_raw[];
    unsigned char* smem = fg_raw + ((1024u - (t5_smem(fg_raw) & 1023u)) & 1023u);
    unsigned long long* full = reinterpret_cast<unsigned long long*>(smem + S::STAGES * S::STAGE);
    unsigned long long* empty = full + S::STAGES;
    unsigned long long* acc_full = empty + S::STAGES;
    unsigned* tmem_slot = reinterpret_cast<unsigned*>(acc_full + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x, nsplit = gridDim.x;
    const int64_t n0 = (int64_t)blockIdx.y * FG_ROWS, m0 = (int64_t)blockIdx.z * NT;
    const int s0 = (int)((int64_t)a.slabs * split / nsplit), s1 = (int)((int64_t)a.slabs * (split + 1) / nsplit);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            t5_bar_init(t5_smem(full + s), 1);
            t5_bar_init(t5_smem(empty + s), 1);
        }
        t5_bar_init(t5_smem(acc_full), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(t5_smem(tmem_slot)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    t5_fence_before();
    __syncthreads();
    t5_fence_after();
    const unsigned tmem = *tmem_slot;

    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            const uint8_t* ws = a.w_scales + (int64_t)blockIdx.y * a.tiles * 512;
            const uint8_t* xs = a.x_scales + (m0 >> 7) * a.tiles * 512;
            int i = 0;
            for (; i < s1 - s0; ++i) {
                const int s = i % S::STAGES;
                if (!t5_bar_wait(t5_smem(empty + s), ((unsigned)(i / S::STAGES) & 1u) ^ 1u, abort_flag)) break;
                const int slab = s0 + i;
                const int64_t atom = (int64_t)slab * S::ATOMS;
                const unsigned sbytes = (unsigned)min((int64_t)S::ATOMS, a.tiles - atom) * 512u;
                const unsigned bar = t5_smem(full + s), at = t5_smem(smem + s * S::STAGE);
                t5_bar_expect(bar, (unsigned)(S::W_BYTES + S::X_BYTES) + 2 * sbytes);
                t5_load_2d(at, &wmap, slab * 128, (int)n0, bar);
                t5_load_2d(at + S::W_BYTES, &xmap, slab * 128, (int)m0, bar);
                t5_load_bulk(at + S::W_BYTES + S::X_BYTES, ws + atom * 512, sbytes, bar);
                t5_load_bulk(at + S::W_BYTES + S::X_BYTES + S::S_BYTES, xs + atom * 512, sbytes, bar);
            }
            for (int j = max(0, i - S::STAGES); j < i; ++j)
                t5_bar_drain(t5_smem(full + j % S::STAGES), (unsigned)(j / S::STAGES) & 1u);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            for (int i = 0; i < s1 - s0; ++i) {
                const int s = i % S::STAGES;
                ok = t5_bar_wait(t5_smem(full + s), (unsigned)(i / S::STAGES) & 1u, abort_flag);
                if (!ok) break;
                t5_fence_after();
                const unsigned at = t5_smem(smem + s * S::STAGE);
                const unsigned sw = at + S::W_BYTES + S::X_BYTES, sx = sw + S::S_BYTES;
                // the stage's own scale columns: free, since the stage was given back
                const unsigned tw = tmem + S::D_COLS + s * S::SF_COLS, tx = tw + S::SF_COLS / 2;
                const int steps = min(4, a.k64 - 4 * (s0 + i));
                const int atoms = FORMAT == SB_FP4_MX ? (steps + 1) / 2 : steps;
                for (int c = 0; c < atoms; ++c) {
                    fg_copy_scales(tw + 4 * c, sw + 512 * c);
                    fg_copy_scales(tx + 4 * c, sx + 512 * c);
                }
                for (int k = 0; k < steps; ++k) {
                    const int c = FORMAT == SB_FP4_MX ? k >> 1 : k;
                    fg_mma<FORMAT>(tmem, t5_desc_sw128(at + 32 * k), t5_desc_sw128(at + S::W_BYTES + 32 * k),
                                   fg_idesc<FORMAT>(FG_ROWS, NT, FORMAT == SB_FP4_MX ? k & 1 : 0), tw + 4 * c, tx + 4 * c, i > 0 || k > 0);
                }
                fg_commit(t5_smem(empty + s));
            }
            fg_commit(t5_smem(acc_full));
        }
    } else {
        ok = __all_sync(0xffffffffu, t5_bar_wait(t5_smem(acc_full), 0u, abort_flag));
        t5_fence_after();
        const int q = warp & 3;                                      // the warp's quarter of the lanes
        const int64_t n = n0 + q * 32 + lane;
        const float alpha = (a.w_tensor ? __ldg(a.w_tensor) : 1.f) * (a.x_tensor ? __ldg(a.x_tensor) : 1.f);
        const int ntok = (int)min((int64_t)NT, a.M - m0);
        float* part = reinterpret_cast<float*>(smem);               // [token][128], the ring is done with
        if (ok) {
#pragma unroll
            for (int c = 0; c < NT; c += 16) {
                if (c >= ntok) break;
                unsigned r[16];
                t5_ld16(tmem + ((unsigned)(q * 32) << 16) + (unsigned)c, r);
                t5_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    if (c + k < ntok) {
                        if (nsplit > 1) part[(c + k) * FG_ROWS + q * 32 + lane] = __uint_as_float(r[k]);
                        else if (n < a.N) fg_store(a, m0 + c + k, n, alpha * __uint_as_float(r[k]));
                    }
                }
            }
        }
        t5_fence_before();
    }
    __syncwarp();
    if (nsplit > 1) {
        // the segments of this tile are the CTAs of one cluster: every CTA adds a part of the tile's
        // outputs over all segments, in their order, out of their shared memory
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const float* part = reinterpret_cast<const float*>(smem);
        const float* seg[FG_MAX_SPLIT];
#pragma unroll
        for (int s = 0; s < FG_MAX_SPLIT; ++s) seg[s] = cluster.map_shared_rank(part, s < nsplit ? s : 0);
        const float alpha = (a.w_tensor ? __ldg(a.w_tensor) : 1.f) * (a.x_tensor ? __ldg(a.x_tensor) : 1.f);
        const int total = (int)min((int64_t)NT, a.M - m0) * FG_ROWS;
        const bool fine = *abort_flag == 0;
        for (int idx = split * FG_THREADS + threadIdx.x; idx < total; idx += nsplit * FG_THREADS) {
            float v[FG_MAX_SPLIT];
#pragma unroll
            for (int s = 0; s < FG_MAX_SPLIT; ++s) v[s] = s < nsplit ? seg[s][idx] : 0.f;
            float sum = v[0];
#pragma unroll
            for (int s = 1; s < FG_MAX_SPLIT; ++s)
                if (s < nsplit) sum += v[s];
            const int64_t n = n0 + (idx & (FG_ROWS - 1));
            if (fine && n < a.N) fg_store(a, m0 + idx / FG_ROWS, n, alpha * sum);
        }
        cluster.sync();                              // nobody leaves while its sums may still be read
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        t5_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
    }
    if (threadIdx.x == 0 && *abort_flag) sb_latch(a.st, SB_ERR_TIMEOUT, SBK_FP4);
}

template <int FORMAT, int NT>
sb_status fg_tile_launch(sb_ctx* ctx, const FgArgs& a, const uint8_t* w_codes, const uint8_t* x_codes, int64_t K) {
    using S = FgShape<FORMAT, NT>;
    CUtensorMap wmap, xmap;
    const int64_t pitch = fp4_padded_cols(K) / 2;
    sb_status st = t5_map_rows(ctx, &wmap, w_codes, a.N, pitch, pitch, FG_ROWS);
    if (st == SB_OK) st = t5_map_rows(ctx, &xmap, x_codes, a.M, pitch, pitch, NT);
    if (st != SB_OK) return st;
    auto* kernel = fp4_tile_kernel<FORMAT, NT>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (a.N + FG_ROWS - 1) / FG_ROWS, tok_tiles = (a.M + NT - 1) / NT;
    if (row_tiles > 65535 || tok_tiles > 65535) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 gemm: too many tiles");
    // segments of the columns: about two CTAs per SM, of at least two slabs each
    int64_t split = 2 * (int64_t)ctx->sm_count / (row_tiles * tok_tiles);
    if (split > a.slabs / 2) split = a.slabs / 2;
    if (split > FG_MAX_SPLIT) split = FG_MAX_SPLIT;
    if (split < 1) split = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)split, (unsigned)row_tiles, (unsigned)tok_tiles);
    cfg.blockDim = dim3(FG_THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, wmap, xmap, a));
    SB_LAUNCHED(ctx);
    return SB_OK;
}

template <int FORMAT>
sb_status fg_launch(sb_ctx* ctx, const FgArgs& a, const uint8_t* w_codes, const uint8_t* x_codes, int64_t K) {
    return a.M <= 16 ? fg_tile_launch<FORMAT, 16>(ctx, a, w_codes, x_codes, K)
         : a.M <= 32 ? fg_tile_launch<FORMAT, 32>(ctx, a, w_codes, x_codes, K)
         : a.M <= 64 ? fg_tile_launch<FORMAT, 64>(ctx, a, w_codes, x_codes, K) : fg_tile_launch<FORMAT, 128>(ctx, a, w_codes, x_codes, K);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

extern "C" sb_status sb_fp4_gemm(sb_ctx* ctx, const uint8_t* a_codes, const uint8_t* a_scales, const float* a_tensor_scale,
                                 int64_t M, const uint8_t* b_codes, const uint8_t* b_scales, const float* b_tensor_scale,
                                 int64_t N, int64_t K, int format, void* Y, int out_f32, int64_t ldy) {
    if (!ctx) return SB_ERR_INVALID;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !Y || M <= 0 || N <= 0 || K <= 0)
        return sb_fail(ctx, SB_ERR_INVALID, "fp4 gemm: null or empty");
    if (format != SB_FP4_MX && format != SB_FP4_NV) return sb_fail(ctx, SB_ERR_INVALID, "fp4 gemm: unknown format %d", format);
    if (format == SB_FP4_MX && (a_tensor_scale || b_tensor_scale))
        return sb_fail(ctx, SB_ERR_INVALID, "fp4 gemm: SB_FP4_MX has no tensor scale");
    if (ldy < N || !aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) ||
        (reinterpret_cast<uintptr_t>(Y) & (out_f32 ? 3 : 1)))
        return sb_fail(ctx, SB_ERR_SHAPE, "fp4 gemm: ldy >= N and 16-byte aligned codes and scales");
    if (M >= (1ll << 30) || N >= (1ll << 30) || K >= (1ll << 30)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 gemm: sizes must fit 30 bits");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    FgArgs a{};
    a.w_scales = b_scales; a.x_scales = a_scales;
    a.w_tensor = b_tensor_scale; a.x_tensor = a_tensor_scale;
    a.tiles = fp4_scale_tiles(K, format);
    a.M = M; a.N = N;
    a.slabs = (int)((fp4_padded_cols(K) + FG_SLAB - 1) / FG_SLAB);
    a.k64 = (int)((fp4_padded_cols(K) + 63) / 64);
    a.Y = Y; a.ldy = ldy; a.out_f32 = out_f32 ? 1 : 0;
    a.st = ctx->dstate;
    return format == SB_FP4_MX ? fg_launch<SB_FP4_MX>(ctx, a, b_codes, a_codes, K) : fg_launch<SB_FP4_NV>(ctx, a, b_codes, a_codes, K);
}
