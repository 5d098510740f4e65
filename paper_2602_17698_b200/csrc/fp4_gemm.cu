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
// Bound by the latency of its rings: 1 token 4096 -> 4096 10.3 us and 24 tokens 4096 -> 14336 (MX) 12.4 us,
// 4 to 5 us of which quantise the tokens; the weights come at 2.7 TB/s in the second.
// fp4_pair_kernel: two CTAs on tiles of 256 weight rows x 256 tokens, which halves what a CTA copies for a product. 8192
// tokens 4096 -> 14336 (NV) 209 to 224 us, 4.3 to 4.6 PFLOP/s, where the power limit holds the clock down (tensor
// pipe 68 % active; without the scale copies 5 to 12 % less time); 500 tokens 14336 -> 4096 27 us.
#include <cooperative_groups.h>

#include "fp4.cuh"
#include "tensor5.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int FG_ROWS = 128;             // weight rows of a tile
constexpr int FG_SLAB = 256;             // columns per ring stage: 128 bytes of codes
// More tokens than this: pairs of CTAs. 4096 -> 4096, pairs and single CTAs: 192 tokens 18.5 and 15.1 us, 257 20.6 and
// 18.5, 384 20.6 and 26.7, 512 20.6 and 22.5; 4096 -> 14336: 129 18.5 and 17.8, 257 26.7 and 24.6, 512 27.7 and 28.8.
constexpr int FG_PAIR_FROM = 256;
constexpr int FG_MAX_SPLIT = 8;          // portable cluster size
constexpr int FG_THREADS = 192;          // warp 0: copies, warp 1: products, warps 2-5: results

struct FgArgs {
    const float *w_tensor, *x_tensor;    // or NULL
    int64_t M, N;                        // tokens, weight rows
    int slabs, k64;                      // ring stages and instruction steps along K
    int row_tiles, tiles;                // fp4_pair_kernel: tiles of 256 weight rows, tiles in all
    void* Y;
    int64_t ldy;
    int out_f32;
    SbDeviceState* st;
};
// codes and scales of weights and tokens
struct FgMaps { CUtensorMap w, x, ws, xs; };

template <int FORMAT, int NT>
struct FgShape {
    static constexpr int ATOMS = FORMAT == SB_FP4_MX ? 2 : 4;        // scale tiles of a slab
    static constexpr int W_BYTES = FG_ROWS * 128, X_BYTES = NT * 128, S_BYTES = ATOMS * 512;
    static constexpr int STAGE = W_BYTES + X_BYTES + 2 * S_BYTES;
    static constexpr int STAGES = NT <= 32 ? 4 : 3;                  // two CTAs per SM
    static constexpr int SMEM = STAGES * STAGE + 1024 + 256;
    static constexpr int SF_COLS = 2 * 4 * ATOMS;                    // scale columns of a stage
    static constexpr int D_COLS = NT < 32 ? 32 : NT;
    static constexpr int TMEM = D_COLS + STAGES * SF_COLS <= 128 ? 128 : 256;
    static_assert(D_COLS + STAGES * SF_COLS <= 256 && SMEM + 1024 <= 227 * 512, "two CTAs of an SM");
    static_assert(FG_ROWS * NT * 4 <= STAGES * STAGE, "partial sums fit where the ring was");
};

// Instruction descriptor: e2m1 x e2m1, both K-major, M = m, N = n, the scale format, and which half
// of a 32-bit scale cell the step reads (MX keeps two steps' scales in a cell).
template <int FORMAT>
__device__ __forceinline__ constexpr unsigned fg_idesc(int m, int n, int half) {
    return 1u << 7 | 1u << 10 | (unsigned)(n >> 3) << 17 | (FORMAT == SB_FP4_MX ? 1u << 23 : 0u) | (unsigned)(m >> 7) << 27 |
           (unsigned)(2 * half) << 4 | (unsigned)(2 * half) << 29;
}
// issued by one lane of a converged warp; PAIR: by the leader of a pair of CTAs, for both
template <int FORMAT, bool PAIR>
__device__ __forceinline__ void fg_mma(bool one, unsigned d, unsigned long long a, unsigned long long b, unsigned idesc,
                                       unsigned sa, unsigned sb, unsigned accumulate) {
#define FG_MMA(GROUP, KIND)                                                                                              \
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %7, 0;\n\t"                          \
                 "@q tcgen05.mma.cta_group::" GROUP "." KIND " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"                    \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "r"((unsigned)one) : "memory")
    if (FORMAT == SB_FP4_MX && PAIR) FG_MMA("2", "kind::mxf4.block_scale.scale_vec::2X");
    else if (FORMAT == SB_FP4_MX) FG_MMA("1", "kind::mxf4.block_scale.scale_vec::2X");
    else if (PAIR) FG_MMA("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
    else FG_MMA("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
#undef FG_MMA
}
template <bool PAIR>
__device__ __forceinline__ void fg_copy_scales(bool one, unsigned taddr, unsigned smem) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}"
                     ::"r"(taddr), "l"(t5_desc_rows16(smem)), "r"((unsigned)one) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
                     ::"r"(taddr), "l"(t5_desc_rows16(smem)), "r"((unsigned)one) : "memory");
}
// the barrier (PAIR: of the CTAs in the mask) is arrived on when everything issued so far is done
template <bool PAIR>
__device__ __forceinline__ void fg_commit(bool one, unsigned bar, unsigned ctas = 0) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
                     "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                     ::"r"(bar), "h"((unsigned short)ctas), "r"((unsigned)one) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                     "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                     ::"r"(bar), "r"((unsigned)one) : "memory");
}
template <typename OUT>
__device__ __forceinline__ void fg_put(OUT* p, float v);
template <> __device__ __forceinline__ void fg_put(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void fg_put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
// COLS columns (tokens) of one weight row: p, then every ldy; n of them exist
template <typename OUT, int COLS>
__device__ __forceinline__ void fg_store_row(OUT* p, int64_t ldy, const unsigned (&r)[COLS], float alpha, int n) {
    if (n >= COLS) {
#pragma unroll
        for (int k = 0; k < COLS; ++k, p += ldy) fg_put(p, alpha * __uint_as_float(r[k]));
    } else {
#pragma unroll
        for (int k = 0; k < COLS; ++k, p += ldy)
            if (k < n) fg_put(p, alpha * __uint_as_float(r[k]));
    }
}
template <int COLS>
__device__ __forceinline__ void fg_store_columns(const FgArgs& a, int64_t m, int64_t n, const unsigned (&r)[COLS], float alpha, int count) {
    if (a.out_f32) fg_store_row(static_cast<float*>(a.Y) + m * a.ldy + n, a.ldy, r, alpha, count);
    else fg_store_row(static_cast<__nv_bfloat16*>(a.Y) + m * a.ldy + n, a.ldy, r, alpha, count);
}
__device__ __forceinline__ float fg_alpha(const FgArgs& a) {
    return (a.w_tensor ? __ldg(a.w_tensor) : 1.f) * (a.x_tensor ? __ldg(a.x_tensor) : 1.f);
}

template <int FORMAT, int NT>
__global__ void __launch_bounds__(FG_THREADS)
fp4_tile_kernel(const __grid_constant__ FgMaps maps, const FgArgs a) {
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
    const unsigned tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);

    bool ok = true;
    if (warp == 0) {
        const bool one = t5_elect();
        int i = 0;
        for (; i < s1 - s0; ++i) {
            const int s = i % S::STAGES;
            if (!__all_sync(0xffffffffu, t5_bar_wait(t5_smem(empty + s), ((unsigned)(i / S::STAGES) & 1u) ^ 1u, abort_flag))) break;
            const int slab = s0 + i;
            const unsigned bar = t5_smem(full + s), at = t5_smem(smem + s * S::STAGE);
            if (one) {
                t5_bar_expect(bar, (unsigned)S::STAGE);
                t5_load_2d(at, &maps.w, slab * 128, (int)n0, bar);
                t5_load_2d(at + S::W_BYTES, &maps.x, slab * 128, (int)m0, bar);
                t5_load_2d(at + S::W_BYTES + S::X_BYTES, &maps.ws, slab * (S::S_BYTES / 8), (int)blockIdx.y, bar);
                t5_load_2d(at + S::W_BYTES + S::X_BYTES + S::S_BYTES, &maps.xs, slab * (S::S_BYTES / 8), (int)(m0 >> 7), bar);
            }
            __syncwarp();
        }
        for (int j = max(0, i - S::STAGES); j < i; ++j)
            t5_bar_drain(t5_smem(full + j % S::STAGES), (unsigned)(j / S::STAGES) & 1u);
    } else if (warp == 1) {
        const bool one = t5_elect();
        for (int i = 0; i < s1 - s0; ++i) {
            const int s = i % S::STAGES;
            ok = __all_sync(0xffffffffu, t5_bar_wait(t5_smem(full + s), (unsigned)(i / S::STAGES) & 1u, abort_flag));
            if (!ok) break;
            t5_fence_after();
            const unsigned at = t5_smem(smem + s * S::STAGE);
            const unsigned sw = at + S::W_BYTES + S::X_BYTES, sx = sw + S::S_BYTES;
            // the stage's own scale columns: free, since the stage was given back
            const unsigned tw = tmem + S::D_COLS + s * S::SF_COLS, tx = tw + S::SF_COLS / 2;
            const int steps = min(4, a.k64 - 4 * (s0 + i));
#pragma unroll
            for (int c = 0; c < S::ATOMS; ++c) {
                fg_copy_scales<false>(one, tw + 4 * c, sw + 512 * c);
                fg_copy_scales<false>(one, tx + 4 * c, sx + 512 * c);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = FORMAT == SB_FP4_MX ? k >> 1 : k;
                fg_mma<FORMAT, false>(one && k < steps, tmem, t5_desc_sw128(at + 32 * k), t5_desc_sw128(at + S::W_BYTES + 32 * k),
                                      fg_idesc<FORMAT>(FG_ROWS, NT, FORMAT == SB_FP4_MX ? k & 1 : 0), tw + 4 * c, tx + 4 * c, i > 0 || k > 0);
            }
            fg_commit<false>(one, t5_smem(empty + s));
        }
        fg_commit<false>(one, t5_smem(acc_full));
    } else {
        ok = __all_sync(0xffffffffu, t5_bar_wait(t5_smem(acc_full), 0u, abort_flag));
        t5_fence_after();
        const int q = warp & 3;                                      // the warp's quarter of the lanes
        const int64_t n = n0 + q * 32 + lane;
        const float alpha = fg_alpha(a);
        const int ntok = (int)min((int64_t)NT, a.M - m0);
        float* part = reinterpret_cast<float*>(smem) + q * 32 + lane;      // [token][128], the ring is done with
        if (ok) {
#pragma unroll 1
            for (int c = 0; c < ntok; c += 32) {
                unsigned r[32];
                t5_ld32(tmem + ((unsigned)(q * 32) << 16) + (unsigned)c, r);
                t5_wait_ld();
                if (nsplit > 1) {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (NT >= 32 || k < NT) part[(c + k) * FG_ROWS] = __uint_as_float(r[k]);
                } else if (n < a.N) fg_store_columns(a, m0 + c, n, r, alpha, ntok - c);
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
        const float alpha = fg_alpha(a);
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
            const int64_t n = n0 + (idx & (FG_ROWS - 1)), m = m0 + idx / FG_ROWS;
            if (fine && n < a.N) {
                if (a.out_f32) fg_put(static_cast<float*>(a.Y) + m * a.ldy + n, alpha * sum);
                else fg_put(static_cast<__nv_bfloat16*>(a.Y) + m * a.ldy + n, alpha * sum);
            }
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

// ---- many tokens: pairs of CTAs ------------------------------------------------------------------
template <int FORMAT>
struct FpShape {
    static constexpr int TOKENS = 256;                               // of a tile; its weight rows: 256
    static constexpr int ATOMS = FORMAT == SB_FP4_MX ? 2 : 4;
    static constexpr int HALF = 128 * 128;                           // this CTA's 128 rows of an operand
    static constexpr int S_BYTES = ATOMS * 512;
    static constexpr int STAGE = 2 * HALF + 3 * S_BYTES;             // scales: its weight rows', all tokens'
    static constexpr int STAGES = 5;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 256;
    static constexpr int TMEM = 512;
    static constexpr int ACC = 160;                                  // second accumulator's first column
    static constexpr int BOTH = TOKENS - ACC;                        // columns that both accumulators use
    static constexpr int SF = ACC + TOKENS;                          // scales: of two slabs, 24 columns each half of a slab
    static constexpr int EPI_WARPS = 8;
    static constexpr int THREADS = (2 + EPI_WARPS) * 32;
};

// Copies of a pair count their bytes on the leader's barrier (a cluster address).
__device__ __forceinline__ void fp_load(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}

// SPLIT: a tile per cluster, its columns cut into segments, one per pair of the cluster's CTAs, added in
// segment order through distributed shared memory.
template <int FORMAT, bool SPLIT>
__global__ void __launch_bounds__(FpShape<FORMAT>::THREADS, 1)
fp4_pair_kernel(const __grid_constant__ FgMaps maps, const FgArgs a) {
    using S = FpShape<FORMAT>;
    extern __shared__ unsigned char fg_raw[];
    unsigned char* smem = fg_raw + ((1024u - (t5_smem(fg_raw) & 1023u)) & 1023u);
    unsigned long long* full = reinterpret_cast<unsigned long long*>(smem + S::STAGES * S::STAGE);
    unsigned long long* empty = full + S::STAGES;
    unsigned long long* acc_full = empty + S::STAGES;                // [2]
    unsigned long long* acc_free = acc_full + 2;                     // the columns both accumulators use
    unsigned* tmem_slot = reinterpret_cast<unsigned*>(acc_free + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned crank = t5_cta_rank(), rank = crank & 1, leader = crank & ~1u;       // rank 0 of a pair leads it
    const unsigned both = 3u << leader;
    const int segs = SPLIT ? (int)t5_cluster_size() / 2 : 1, seg = SPLIT ? (int)(crank >> 1) : 0;
    const int pair = (int)(blockIdx.x >> 1) / segs, pairs = (int)(gridDim.x >> 1) / segs;
    const int s0 = SPLIT ? (int)((int64_t)a.slabs * seg / segs) : 0, s1 = SPLIT ? (int)((int64_t)a.slabs * (seg + 1) / segs) : a.slabs;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            t5_bar_init(t5_smem(full + s), 1);
            t5_bar_init(t5_smem(empty + s), 1);
        }
        t5_bar_init(t5_smem(acc_full), 1);
        t5_bar_init(t5_smem(acc_full + 1), 1);
        t5_bar_init(t5_smem(acc_free), 2 * S::EPI_WARPS);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(t5_smem(tmem_slot)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    t5_fence_before();
    t5_cluster_sync();                       // the barriers of both CTAs exist before anything arrives on them
    t5_fence_after();
    const unsigned tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);

    if (warp == 0) {
        const bool one = t5_elect();
        int i = 0;                                                   // ring stages filled, over all tiles
        bool ok = true;
        for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
            const int rt = tile % a.row_tiles, tt = tile / a.row_tiles;
            const int n0 = rt * 256 + (int)rank * 128, m0 = tt * S::TOKENS + (int)rank * 128;
            for (int slab = s0; slab < s1; ++slab, ++i) {
                const int s = i % S::STAGES;
                ok = __all_sync(0xffffffffu, t5_bar_wait(t5_smem(empty + s), ((unsigned)(i / S::STAGES) & 1u) ^ 1u, abort_flag));
                if (!ok) break;
                const unsigned at = t5_smem(smem + s * S::STAGE), bar = t5_cluster_addr(t5_smem(full + s), leader);
                if (one) {
                    if (rank == 0) t5_bar_expect(t5_smem(full + s), 2u * S::STAGE);
                    fp_load(at, &maps.w, slab * 128, n0, bar);
                    fp_load(at + S::HALF, &maps.x, slab * 128, m0, bar);
                    fp_load(at + 2 * S::HALF, &maps.ws, slab * (S::S_BYTES / 8), n0 >> 7, bar);
                    fp_load(at + 2 * S::HALF + S::S_BYTES, &maps.xs, slab * (S::S_BYTES / 8), tt * 2, bar);
                }
                __syncwarp();
            }
        }
        // bytes of both CTAs are counted by the leader: it waits for what is still in flight
        if (rank == 0)
            for (int j = max(0, i - S::STAGES); j < i; ++j)
                t5_bar_drain(t5_smem(full + j % S::STAGES), (unsigned)(j / S::STAGES) & 1u);
    } else if (warp == 1) {
        if (rank == 0) {
            const bool one = t5_elect();
            int i = 0, n = 0;                                        // stages and tiles so far
            bool ok = true;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs, ++n) {
                // the epilogue has read the columns this accumulator shares with the last tile's, and
                // with that everything of the tile before
                if (n > 0) ok = __all_sync(0xffffffffu, t5_bar_wait(t5_smem(acc_free), (unsigned)(n - 1) & 1u, abort_flag));
                if (!ok) break;
                t5_fence_after();
                const unsigned acc = tmem + (unsigned)((n & 1) * S::ACC);
                for (int slab = s0; slab < s1; ++slab, ++i) {
                    const int s = i % S::STAGES;
                    // the scales of two slabs ago are done with (products are not ordered before later copies);
                    // then this slab's copies, which the products are waiting for
                    ok = i < 2 || t5_bar_wait(t5_smem(empty + (i - 2) % S::STAGES), (unsigned)((i - 2) / S::STAGES) & 1u, abort_flag);
                    ok = __all_sync(0xffffffffu, ok && t5_bar_wait(t5_smem(full + s), (unsigned)(i / S::STAGES) & 1u, abort_flag));
                    if (!ok) break;
                    t5_fence_after();
                    const unsigned at = t5_smem(smem + s * S::STAGE);
                    const unsigned sw = at + 2 * S::HALF, sx = sw + S::S_BYTES;
                    const int steps = min(4, a.k64 - 4 * slab);
                    // two scale tiles at a time (MX: the whole slab's)
#pragma unroll
                    for (int h = 0; h < S::ATOMS / 2; ++h) {
                        const unsigned area = tmem + S::SF + 48u * (unsigned)(i & 1) + 24u * (unsigned)h;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            fg_copy_scales<true>(one, area + 4 * c, sw + 512 * (2 * h + c));
                            fg_copy_scales<true>(one, area + 8 + 8 * c, sx + 512 * (2 * h + c));
                            fg_copy_scales<true>(one, area + 12 + 8 * c, sx + S::S_BYTES + 512 * (2 * h + c));
                        }
                        constexpr int KS = FORMAT == SB_FP4_MX ? 4 : 2;
#pragma unroll
                        for (int k = KS * h; k < KS * (h + 1); ++k) {
                            const int c = FORMAT == SB_FP4_MX ? k >> 1 : k & 1;
                            fg_mma<FORMAT, true>(one && k < steps, acc, t5_desc_sw128(at + 32 * k), t5_desc_sw128(at + S::HALF + 32 * k),
                                                 fg_idesc<FORMAT>(256, S::TOKENS, FORMAT == SB_FP4_MX ? k & 1 : 0), area + 4 * c,
                                                 area + 8 + 8 * c, slab > s0 || k > 0);
                        }
                    }
                    fg_commit<true>(one, t5_smem(empty + s), both);
                }
                fg_commit<true>(one, t5_smem(acc_full + (n & 1)), both);
            }
        }
    } else {
        // warp: a quarter of the lanes, half of the columns; first its part of the columns that the
        // next tile's accumulator needs, then the rest
        const int q = warp & 3, half = (warp - 2) >> 2;
        const unsigned free_leader = t5_cluster_addr(t5_smem(acc_free), leader);
        const float alpha = fg_alpha(a);
        int n = 0;
        for (int tile = pair; tile < a.tiles; tile += pairs, ++n) {
            const int rt = tile % a.row_tiles, tt = tile / a.row_tiles;
            const int b = n & 1;
            if (!__all_sync(0xffffffffu, t5_bar_wait(t5_smem(acc_full + b), (unsigned)(n >> 1) & 1u, abort_flag))) break;
            t5_fence_after();
            const int64_t m0 = (int64_t)tt * S::TOKENS, row = (int64_t)rt * 256 + rank * 128 + q * 32 + lane;
            const int ntok = (int)min((int64_t)S::TOKENS, a.M - m0);
            const unsigned src = tmem + ((unsigned)(q * 32) << 16) + (unsigned)(b * S::ACC);
            // columns in pieces of 16: BOTH / 32 of the shared ones (the end of the first accumulator, the
            // start of the second), then ACC / 32 of the others
#pragma unroll 1
            for (int u = 0; u < S::TOKENS / 32; ++u) {
                const bool shared_part = u < S::BOTH / 32;
                const int c = shared_part ? (b ? 0 : S::ACC) + (half * (S::BOTH / 32) + u) * 16
                                          : (b ? S::BOTH : 0) + (half * (S::ACC / 32) + u - S::BOTH / 32) * 16;
                unsigned r[16];
                t5_ld16(src + (unsigned)c, r);
                t5_wait_ld();
                if (u == S::BOTH / 32 - 1) {
                    t5_fence_before();
                    __syncwarp();
                    if (lane == 0)
                        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(free_leader) : "memory");
                }
                if (SPLIT) {
                    float* part = reinterpret_cast<float*>(smem) + c * 128 + q * 32 + lane;    // [token][128], the ring is done with
#pragma unroll
                    for (int k = 0; k < 16; ++k) part[k * 128] = __uint_as_float(r[k]);
                } else if (row < a.N) fg_store_columns(a, m0 + c, row, r, alpha, ntok - c);
                __syncwarp();
            }
        }
    }
    if (SPLIT) {
        // every CTA adds the segments of its rows over its share of the tokens
        __syncwarp();
        t5_fence_before();
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const int rt = pair % a.row_tiles, tt = pair / a.row_tiles;
        const float* part = reinterpret_cast<const float*>(smem);
        const float* from[FG_MAX_SPLIT / 2];
#pragma unroll
        for (int g = 0; g < FG_MAX_SPLIT / 2; ++g) from[g] = cluster.map_shared_rank(part, 2 * (g < segs ? g : 0) + (int)rank);
        const float alpha = fg_alpha(a);
        const int64_t m0 = (int64_t)tt * S::TOKENS, n0 = (int64_t)rt * 256 + rank * 128;
        const int ntok = (int)min((int64_t)S::TOKENS, a.M - m0);
        const int t0 = ntok * seg / segs, t1 = ntok * (seg + 1) / segs;
        const bool fine = *abort_flag == 0;
#pragma unroll 4
        for (int idx = t0 * 128 + (int)threadIdx.x; idx < t1 * 128; idx += S::THREADS) {
            float sum = from[0][idx];
#pragma unroll
            for (int g = 1; g < FG_MAX_SPLIT / 2; ++g)
                if (g < segs) sum += from[g][idx];
            const int64_t n = n0 + (idx & 127), m = m0 + idx / 128;
            if (fine && n < a.N) {
                if (a.out_f32) fg_put(static_cast<float*>(a.Y) + m * a.ldy + n, alpha * sum);
                else fg_put(static_cast<__nv_bfloat16*>(a.Y) + m * a.ldy + n, alpha * sum);
            }
        }
    }
    __syncwarp();
    t5_fence_before();
    t5_cluster_sync();                       // nobody leaves while its partner may still use its memory or barriers
    if (warp == 1) {
        t5_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
    }
    if (threadIdx.x == 0 && *abort_flag) sb_latch(a.st, SB_ERR_TIMEOUT, SBK_FP4);
}

struct FgOperand { const uint8_t *codes, *scales; };

// maps of codes (boxes of 256 columns) and scales (the tiles of 256 columns of box_tiles row tiles)
sb_status fg_maps(sb_ctx* ctx, FgMaps* m, const FgArgs& a, const FgOperand& w, const FgOperand& x, int64_t K, int format,
                  int x_box, int x_scale_box) {
    const int64_t pitch = fp4_padded_cols(K) / 2, tiles = fp4_scale_tiles(K, format);
    const int box = (format == SB_FP4_MX ? 2 : 4) * 64;             // 8-byte elements of a slab's scales
    constexpr auto U64 = CU_TENSOR_MAP_DATA_TYPE_UINT64;
    sb_status st = t5_map_rows(ctx, &m->w, w.codes, a.N, pitch, FG_ROWS);
    if (st == SB_OK) st = t5_map_rows(ctx, &m->x, x.codes, a.M, pitch, x_box);
    if (st == SB_OK) st = t5_map(ctx, &m->ws, U64, w.scales, (a.N + 127) / 128, tiles * 64, tiles * 512, box, 1, false);
    if (st == SB_OK) st = t5_map(ctx, &m->xs, U64, x.scales, (a.M + 127) / 128, tiles * 64, tiles * 512, box, x_scale_box, false);
    return st;
}

template <int FORMAT, int NT>
sb_status fg_tile_launch(sb_ctx* ctx, const FgArgs& a, const FgOperand& w, const FgOperand& x, int64_t K) {
    using S = FgShape<FORMAT, NT>;
    FgMaps maps;
    const sb_status st = fg_maps(ctx, &maps, a, w, x, K, FORMAT, NT, 1);
    if (st != SB_OK) return st;
    auto* kernel = fp4_tile_kernel<FORMAT, NT>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (a.N + FG_ROWS - 1) / FG_ROWS, tok_tiles = (a.M + NT - 1) / NT;
    if (row_tiles > 65535 || tok_tiles > 65535) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 gemm: too many tiles");
    // Segments of the columns where the tiles leave half of the SMs idle: about two CTAs per SM, of at
    // least four slabs each. The sums of a cluster cost more than half a row of slabs: 4096 -> 14336 (112
    // tiles) takes 23.9 us in two segments and 16.7 in one for 128 tokens, 14.6 and 13.6 for 32; 14336 ->
    // 4096 (32 tiles) 16.5 in eight and 18.5 in four for 64; 4096 -> 4096 12.3 in eight (of two slabs), 10.3 in
    // four for 32.
    const int64_t tiles = row_tiles * tok_tiles;
    int64_t split = 2 * tiles <= ctx->sm_count ? 2 * (int64_t)ctx->sm_count / tiles : 1;
    if (split > a.slabs / 4) split = a.slabs / 4;
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
    SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, maps, a));
    SB_LAUNCHED(ctx);
    return SB_OK;
}

template <int FORMAT, bool SPLIT>
sb_status fg_pair_launch(sb_ctx* ctx, const FgMaps& maps, const FgArgs& a, int64_t pairs, int segs) {
    using S = FpShape<FORMAT>;
    auto* kernel = fp4_pair_kernel<FORMAT, SPLIT>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(2 * pairs * segs));
    cfg.blockDim = dim3(S::THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(2 * segs);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, maps, a));
    SB_LAUNCHED(ctx);
    return SB_OK;
}
template <int FORMAT>
sb_status fg_pairs(sb_ctx* ctx, FgArgs a, const FgOperand& w, const FgOperand& x, int64_t K) {
    using S = FpShape<FORMAT>;
    FgMaps maps;
    const sb_status st = fg_maps(ctx, &maps, a, w, x, K, FORMAT, 128, 2);
    if (st != SB_OK) return st;
    const int64_t row_tiles = (a.N + 255) / 256, tiles = row_tiles * ((a.M + S::TOKENS - 1) / S::TOKENS);
    if (tiles >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "fp4 gemm: too many tiles");
    a.row_tiles = (int)row_tiles;
    a.tiles = (int)tiles;
    // with fewer tiles than half the pairs of SMs the columns are cut too, at least eight slabs a segment
    const int64_t slots = ctx->sm_count / 2;
    int segs = 1;
    while (segs < FG_MAX_SPLIT / 2 && tiles * segs * 2 <= slots && a.slabs >= 16 * segs) segs *= 2;
    if (segs > 1) return fg_pair_launch<FORMAT, true>(ctx, maps, a, tiles, segs);
    return fg_pair_launch<FORMAT, false>(ctx, maps, a, tiles < slots ? tiles : slots, 1);
}

template <int FORMAT>
sb_status fg_launch(sb_ctx* ctx, const FgArgs& a, const FgOperand& w, const FgOperand& x, int64_t K) {
    return a.M <= 16 ? fg_tile_launch<FORMAT, 16>(ctx, a, w, x, K)
         : a.M <= 32 ? fg_tile_launch<FORMAT, 32>(ctx, a, w, x, K)
         : a.M <= 64 ? fg_tile_launch<FORMAT, 64>(ctx, a, w, x, K)
         : a.M <= FG_PAIR_FROM ? fg_tile_launch<FORMAT, 128>(ctx, a, w, x, K) : fg_pairs<FORMAT>(ctx, a, w, x, K);
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
    a.w_tensor = b_tensor_scale; a.x_tensor = a_tensor_scale;
    a.M = M; a.N = N;
    a.slabs = (int)((fp4_padded_cols(K) + FG_SLAB - 1) / FG_SLAB);
    a.k64 = (int)((fp4_padded_cols(K) + 63) / 64);
    a.Y = Y; a.ldy = ldy; a.out_f32 = out_f32 ? 1 : 0;
    a.st = ctx->dstate;
    const FgOperand w{b_codes, b_scales}, x{a_codes, a_scales};
    return format == SB_FP4_MX ? fg_launch<SB_FP4_MX>(ctx, a, w, x, K) : fg_launch<SB_FP4_NV>(ctx, a, w, x, K);
}
