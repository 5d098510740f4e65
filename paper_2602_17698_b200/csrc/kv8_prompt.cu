// Attention of many query rows over the 8-bit cache (prompts and chunks of prompts) on tcgen05.
//
// A CTA takes 256 query rows of one cache head (new tokens x query heads that share it) as two
// tiles of 128, one row per softmax thread, and walks over the keys in tiles of 128:
//     S = Q K^T   (128 x 128, fp16 x fp16 -> fp32 in tensor memory)
//     P = 2^(S factor - m), times the value scale of its 16 keys, to fp16, over S's own columns
//     O += P V    (A from tensor memory, V with d contiguous, fp32 in tensor memory)
// The tensor cores cannot multiply 8-bit by 16-bit operands, so four warps convert a tile of K and
// of V to fp16 (exact) into the 128-byte-swizzled layout the instructions read; 256 rows share the
// conversion. Scales never touch K and V: a scale block is 16 columns of S, its key scale goes
// into the factor of S, its value scale into P.
//
// Warps 0-3 and 4-7: softmax of the two tiles; 8-11: conversion; 12 and 14: their products; 13: copies. A softmax
// step takes half a key tile (64 keys): while it works on one half, the tensor cores multiply the
// other half's weights and put the next tile's scores in their place. The running
// maximum of a row is only moved when it is off by more than 2^8 (P stays below 2^8, far from
// fp16's end), so sums in tensor memory are rarely touched between tiles.
//
// Per 128 keys and 256 rows the products need 2048 cycles and the exponentials 2048 (16 per cycle
// and SM): both bound the kernel.
#include "kv8_attention.cuh"
#include "tensor5.cuh"

namespace {

constexpr int PR_ROWS = 128;             // query rows of a tile; two per CTA
constexpr int PR_KEYS = 128;             // keys of a tile
constexpr int PR_BLOCKS = PR_KEYS / SB_KV8_BLOCK;
constexpr int PR_SUB = 64;               // keys of a softmax step: half a tile
constexpr int PR_SUBBLOCKS = PR_SUB / SB_KV8_BLOCK;
constexpr int PR_THREADS = 16 * 32;       // warp 15 only lends its registers
// registers of a softmax, conversion and other warp's thread: 8 x 184 + 4 x 96 + 4 x 48 warps' shares <= 16 x 128
constexpr int PR_REGS_SOFTMAX = 184, PR_REGS_CONVERT = 96, PR_REGS_REST = 48;
static_assert(8 * PR_REGS_SOFTMAX + 4 * PR_REGS_CONVERT + 4 * PR_REGS_REST <= 16 * 128, "what the block was launched with");
constexpr float PR_SLACK = 8.f;          // log2 of how far a row's maximum may run ahead of its reference

template <int DP>
struct PrShape {
    static constexpr int PANELS = DP / 64;                          // 128-byte columns of an operand row
    static constexpr int PANEL = 128 * 128;                         // bytes: 128 rows x 128
    static constexpr int OPERAND = PANELS * PANEL;
    static constexpr int RING = 3, RAW_RING = 4;                    // converted and raw tiles: K, V, K, V, ...
    static constexpr int RAW = PR_KEYS * DP;
    static constexpr int Q_AT = 0, T_AT = 2 * OPERAND, RAW_AT = T_AT + RING * OPERAND;
    static constexpr int SC_AT = RAW_AT + RAW_RING * RAW;           // scales of four tiles: 8 of K, 8 of V
    static constexpr int BAR_AT = SC_AT + 4 * 64;
    static constexpr int SMEM = BAR_AT + 288 + 1024;
    // tensor memory: S (and P) of the two tiles, then O of the two tiles
    static constexpr int S_COL = 0, O_COL = 256, TMEM = DP == 64 ? 512 : 512;
};

__device__ __forceinline__ void pr_st16(unsigned taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void pr_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// fp16 x fp16 -> fp32, M = 128; A from shared memory (a descriptor) or tensor memory
__device__ __forceinline__ void pr_mma_ss(bool one, unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned acc) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"((unsigned)one) : "memory");
}
__device__ __forceinline__ void pr_mma_ts(bool one, unsigned d, unsigned a, unsigned long long b, unsigned idesc, unsigned acc) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"((unsigned)one) : "memory");
}
__device__ __forceinline__ void pr_commit(bool one, unsigned bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar), "r"((unsigned)one) : "memory");
}
// V [keys][d], d contiguous in panels of 64: 8-key groups 1024 bytes apart, panels PANEL apart
template <int DP>
__device__ __forceinline__ unsigned long long pr_desc_v(unsigned addr) {
    return (unsigned long long)((addr >> 4) & 0x3fffu) | (unsigned long long)(PrShape<DP>::PANEL >> 4) << 16 |
           (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// instruction descriptor: fp32 sums, fp16 operands, M = 128, N = n, B's layout
__device__ __forceinline__ constexpr unsigned pr_idesc(int n, bool b_mn) {
    return 1u << 4 | (b_mn ? 1u << 16 : 0u) | (unsigned)(n >> 3) << 17 | (unsigned)(PR_ROWS >> 4) << 24;
}

// Column c of a row's 64 scores is seen if from < c <= upto; EDGE: some are not.
// Largest score of a row, in units of log2 (kf: factor of each 16 columns, not negative).
template <bool EDGE>
__device__ __forceinline__ float pr_max(unsigned (&s)[PR_SUB / 32][32], const float (&kf)[PR_SUBBLOCKS], int upto, int from) {
    float mx = -INFINITY;
#pragma unroll
    for (int h = 0; h < PR_SUBBLOCKS; ++h) {
        float bm[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = 16 * h + i + u;
                x[u] = __uint_as_float(s[c >> 5][c & 31]);
                if (EDGE && (c > upto || c <= from)) x[u] = -INFINITY;
            }
            bm[0] = fmaxf(fmaxf(bm[0], x[0]), x[1]);
            bm[1] = fmaxf(fmaxf(bm[1], x[2]), x[3]);
        }
        const float top = fmaxf(bm[0], bm[1]);
        // a factor of 0 makes 0 of any score, but no NaN of a block that is masked whole
        mx = fmaxf(mx, EDGE && top == -INFINITY ? -INFINITY : top * kf[h]);
    }
    return mx;
}
// The row's weights 2^(score - ref), times the value scale of their 16 columns, in fp16 over the
// scores; returns the sum of the weights.
template <bool EDGE>
__device__ __forceinline__ float pr_weights(unsigned ts, unsigned (&s)[PR_SUB / 32][32], const float (&kf)[PR_SUBBLOCKS],
                                            const float (&vs)[PR_SUBBLOCKS], float inv, float ref, int upto, int from) {
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < PR_SUB / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float vw = vs[2 * c + h] * inv, kk = kf[2 * c + h];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float e[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    e[u] = at_exp2(fmaf(__uint_as_float(s[c][16 * h + i + u]), kk, -ref));
                    if (EDGE && (32 * c + 16 * h + i + u > upto || 32 * c + 16 * h + i + u <= from)) e[u] = 0.f;
                    sum[u] += e[u];
                }
                p[8 * h + i / 2] = at_half2(e[0] * vw, e[1] * vw);
            }
        }
        pr_st16(ts + 16 * c, p);
    }
    return sum[0] + sum[1];
}

template <int TYPE, int DP>
__global__ void __launch_bounds__(PR_THREADS, 1)
kv8_prompt_kernel(const AtArgs a) {
    using S = PrShape<DP>;
    extern __shared__ unsigned char pr_raw[];
    unsigned char* smem = pr_raw + ((1024u - (t5_smem(pr_raw) & 1023u)) & 1023u);
    float* sc = reinterpret_cast<float*>(smem + S::SC_AT);           // [4][16]
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + S::BAR_AT);
    // raw tiles: landed, converted; converted tiles: there, multiplied; per row tile (and half of a key
    // tile): scores, weights, sums
    unsigned long long *raw_full = bars, *raw_empty = bars + 4, *full = bars + 8, *empty = bars + 12, *sfull = bars + 16,
                       *pfull = bars + 20, *odone = bars + 24, *scfull = bars + 26, *qready = bars + 30, *last = bars + 32;
    unsigned* tmem_slot = reinterpret_cast<unsigned*>(bars + 34);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = blockIdx.x, b = blockIdx.z;
    const int split = (int)(blockIdx.y % (unsigned)a.splits);
    const int rt = a.row_tiles - 1 - (int)(blockIdx.y / (unsigned)a.splits);        // the longest first
    const int D = a.g.dim;
    Kv8Request rq;
    if (!kv8_request(a.g, b, rq, a.st)) return;
    const int rows = rq.n * a.group, r0 = rt * 2 * PR_ROWS;
    if (r0 >= rows) return;
    const int nrow = min(2 * PR_ROWS, rows - r0);
    const bool two = nrow > PR_ROWS;
    const int i0 = r0 / a.group, i1 = (r0 + nrow - 1) / a.group;
    const int hi = rq.past + i1 + 1;
    const int lo = a.window > 0 ? max(0, rq.past + i0 - a.window + 1) & ~(SB_KV8_BLOCK - 1) : 0;
    int chunk = a.chunk;                                             // max_len may be too small: then the chunks grow
    if ((int64_t)chunk * a.splits < hi - lo) chunk = ((hi - lo + a.splits - 1) / a.splits + PR_KEYS - 1) / PR_KEYS * PR_KEYS;
    const int nsplit = (hi - lo + chunk - 1) / chunk;
    const int64_t tile_id = ((int64_t)b * a.g.heads + head) * a.row_tiles + rt;
    if (split >= nsplit) {
        // nothing here: the sum over the chunks skips it
        if (a.splits > 1)
            for (int r = threadIdx.x; r < 2 * PR_ROWS; r += PR_THREADS)
                a.part_ml[(tile_id * a.splits + split) * (2 * PR_ROWS) + r] = make_float2(-INFINITY, 0.f);
        return;
    }
    const int k0 = lo + split * chunk, k1 = min(hi, k0 + chunk);
    const int ntiles = (k1 - k0 + PR_KEYS - 1) / PR_KEYS;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::RAW_RING; ++i) {
            t5_bar_init(t5_smem(raw_full + i), 1);
            t5_bar_init(t5_smem(raw_empty + i), 4);
        }
        for (int i = 0; i < S::RING; ++i) {
            t5_bar_init(t5_smem(full + i), 4);
            t5_bar_init(t5_smem(empty + i), two ? 2 : 1);
        }
        for (int i = 0; i < 4; ++i) {
            t5_bar_init(t5_smem(sfull + i), 1);
            t5_bar_init(t5_smem(pfull + i), 4);
        }
        for (int i = 0; i < 2; ++i) t5_bar_init(t5_smem(odone + i), 1);
        for (int i = 0; i < 4; ++i) t5_bar_init(t5_smem(scfull + i), 1);
        for (int i = 0; i < 2; ++i) {
            t5_bar_init(t5_smem(qready + i), 4);
            t5_bar_init(t5_smem(last + i), 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(t5_smem(tmem_slot)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    t5_fence_before();
    __syncthreads();
    t5_fence_after();
    const unsigned tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    auto wait = [&](unsigned long long* bar, int phase) {
        return (bool)__all_sync(0xffffffffu, t5_bar_wait(t5_smem(bar), (unsigned)phase & 1u, abort_flag));
    };

    if (warp < 8) {
        // ---- softmax: one query row per thread ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PR_REGS_SOFTMAX));
        const int qt = warp >> 2;
        if (qt == 0 || two) {
            const int r = threadIdx.x;                               // row of the CTA
            const int row = r0 + r;
            const bool real = r < nrow;
            float fq;
            {
                const int64_t tok = rq.row0 + (real ? row / a.group : 0);
                const __nv_bfloat16* src = a.q + tok * a.q_token_stride + (int64_t)(head * a.group + (real ? row % a.group : 0)) * a.q_head_stride;
                uint4 x[DP / 8];
                uint32_t m = 0;
#pragma unroll
                for (int c = 0; c < DP / 8; ++c)
                    x[c] = real && 8 * c < D ? *reinterpret_cast<const uint4*>(src + 8 * c) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int c = 0; c < DP / 8; ++c)
                    m = __vmaxu2(m, __vmaxu2(__vmaxu2(x[c].x & 0x7fff7fffu, x[c].y & 0x7fff7fffu), __vmaxu2(x[c].z & 0x7fff7fffu, x[c].w & 0x7fff7fffu)));
                const float up = at_query_scale(max(m & 0xffffu, m >> 16));
                fq = __fdiv_rn(a.scale_log2, up);
                unsigned char* q = smem + S::Q_AT + qt * S::OPERAND + (r & 127) * 128;
#pragma unroll
                for (int c = 0; c < DP / 8; ++c)
                    *reinterpret_cast<uint4*>(q + (c >> 3) * S::PANEL + (((c & 7) ^ (r & 7)) << 4)) =
                        make_uint4(at_half2(bf16lo(x[c].x) * up, bf16hi(x[c].x) * up), at_half2(bf16lo(x[c].y) * up, bf16hi(x[c].y) * up),
                                   at_half2(bf16lo(x[c].z) * up, bf16hi(x[c].z) * up), at_half2(bf16lo(x[c].w) * up, bf16hi(x[c].w) * up));
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(qready + qt));
            }
            const int pos = real ? rq.past + row / a.group : -1;
            // positions of the tile's first and last row decide which key tiles need a mask
            const int pos_lo = rq.past + (r0 + qt * PR_ROWS) / a.group, pos_hi = rq.past + (r0 + min(nrow, (qt + 1) * PR_ROWS) - 1) / a.group;
            const bool ragged = nrow < (qt + 1) * PR_ROWS;
            const unsigned lanes = (unsigned)((warp & 3) * 32) << 16;
            const unsigned ts = tmem + lanes + S::S_COL + qt * 128, to = tmem + lanes + S::O_COL + qt * DP;
            float m = -INFINITY, l = 0.f, vref = 0.f;
            bool ok = true;
            for (int n = 0; n < 2 * ntiles; ++n) {                   // halves of the key tiles
                const int j = n >> 1, u = n & 1;
                ok = wait(sfull + 2 * qt + u, j) && (u || wait(scfull + (j & 3), j >> 2));
                if (!ok) break;
                t5_fence_after();
                unsigned s[PR_SUB / 32][32];
                t5_ld32(ts + PR_SUB * u, s[0]);
                t5_ld32(ts + PR_SUB * u + 32, s[1]);
                const int key = k0 + n * PR_SUB;
                const bool edge = key + PR_SUB > pos_lo + 1 || key + PR_SUB > k1 || ragged || (a.window > 0 && key <= pos_hi - a.window);
                const float* scj = sc + 16 * (j & 3) + PR_SUBBLOCKS * u;
                float kf[PR_SUBBLOCKS], vs[PR_SUBBLOCKS], vmax = 0.f;
#pragma unroll
                for (int i = 0; i < PR_SUBBLOCKS; ++i) {
                    kf[i] = scj[i] * fq;
                    vs[i] = scj[PR_BLOCKS + i];
                    vmax = fmaxf(vmax, vs[i]);
                }
                const int upto = min(pos, k1 - 1) - key, from = a.window > 0 ? pos - a.window - key : -1;
                t5_wait_ld();
                const float mx = edge ? pr_max<true>(s, kf, upto, from) : pr_max<false>(s, kf, upto, from);
                // move the reference (and the power of two of the value scales) when it is too far off
                float f = 1.f;
                if (mx > m + PR_SLACK || (m == -INFINITY && mx > m)) {
                    f = m == -INFINITY ? 0.f : at_exp2(m - mx);
                    m = mx;
                    l *= f;
                }
                if (vmax > vref) {
                    const float fresh = at_value_ref(vmax);
                    f *= __fdiv_rn(vref, fresh);
                    vref = fresh;
                }
                if (n > 0 && __any_sync(0xffffffffu, f != 1.f)) {
                    // the sums so far: the products of the half before this one have to be done
                    ok = wait(odone + qt, n - 1);
                    if (!ok) break;
                    t5_fence_after();
#pragma unroll 1
                    for (int c = 0; c < DP; c += 16) {
                        unsigned o[16];
                        t5_ld16(to + c, o);
                        t5_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        pr_st16(to + c, o);
                    }
                }
                const float inv = at_value_inv(vref), ref = m == -INFINITY ? 0.f : m;
                l += edge ? pr_weights<true>(ts + PR_SUB * u, s, kf, vs, inv, ref, upto, from)
                          : pr_weights<false>(ts + PR_SUB * u, s, kf, vs, inv, ref, upto, from);
                pr_wait_st();
                t5_fence_before();
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(pfull + 2 * qt + u));
            }
            // ---- results ----
            if (ok) ok = wait(odone + qt, 2 * ntiles - 1);
            if (ok) {
                t5_fence_after();
                const int64_t tok = rq.row0 + row / a.group;
                const int h = head * a.group + row % a.group;
                const float norm = a.splits > 1 ? vref : at_norm(l) * vref;
                const int64_t at = (tile_id * a.splits + split) * (2 * PR_ROWS) + r;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    unsigned o[32];
                    t5_ld32(to + c, o);
                    t5_wait_ld();
                    if (real) {
                        if (a.splits > 1) {
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                if (c + i < D)
                                    *reinterpret_cast<float4*>(a.part + at * D + c + i) =
                                        make_float4(__uint_as_float(o[i]) * norm, __uint_as_float(o[i + 1]) * norm,
                                                    __uint_as_float(o[i + 2]) * norm, __uint_as_float(o[i + 3]) * norm);
                        } else {
                            __nv_bfloat16* dst = a.o + tok * a.o_token_stride + h * a.o_head_stride + c;
#pragma unroll
                            for (int i = 0; i < 32; i += 8) {
                                uint32_t w[4];
#pragma unroll
                                for (int u = 0; u < 4; ++u)
                                    w[u] = u32(__floats2bfloat162_rn(__uint_as_float(o[i + 2 * u]) * norm, __uint_as_float(o[i + 2 * u + 1]) * norm));
                                if (c + i < D) *reinterpret_cast<uint4*>(dst + i) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                    __syncwarp();
                }
                if (a.splits > 1) a.part_ml[at] = real ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
                else if (real && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(m, l);
            }
        } else if (a.splits > 1) {
            a.part_ml[(tile_id * a.splits + split) * (2 * PR_ROWS) + threadIdx.x] = make_float2(-INFINITY, 0.f);
        }
    } else if (warp < 12) {
        // ---- conversion: a thread takes one 16-byte piece of every PASS-th row of a tile ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_CONVERT));
        constexpr int PIECES = DP / 16, PASS = 128 / PIECES, NP = PR_KEYS / PASS;
        const int tid = threadIdx.x - 256, piece = tid % PIECES, krow = tid / PIECES;
        // rows from here on were not copied, or hold nothing of the request: zeros
        const int limit = min(rq.len, (k1 + SB_KV8_BLOCK - 1) / SB_KV8_BLOCK * SB_KV8_BLOCK) - k0;
        auto convert = [&](int n) {
            const unsigned src = t5_smem(smem + S::RAW_AT + n % S::RAW_RING * S::RAW) + (unsigned)(krow * D + 16 * piece);
            unsigned char* dst = smem + S::T_AT + n % S::RING * S::OPERAND + (piece >> 2) * S::PANEL;
            const int left = 16 * piece < D ? limit - (n >> 1) * PR_KEYS : 0;
            uint4 x[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                x[i] = make_uint4(0, 0, 0, 0);
                if (krow + PASS * i < left) x[i] = at_lds128(src + (unsigned)(PASS * i * D));
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int kk = krow + PASS * i;
                const uint32_t w[4] = {at_flip<TYPE>(x[i].x), at_flip<TYPE>(x[i].y), at_flip<TYPE>(x[i].z), at_flip<TYPE>(x[i].w)};
                const uint4 lo4 = make_uint4(at_pair<TYPE, 0>(w[0]), at_pair<TYPE, 1>(w[0]), at_pair<TYPE, 0>(w[1]), at_pair<TYPE, 1>(w[1]));
                const uint4 hi4 = make_uint4(at_pair<TYPE, 0>(w[2]), at_pair<TYPE, 1>(w[2]), at_pair<TYPE, 0>(w[3]), at_pair<TYPE, 1>(w[3]));
                const int c = 2 * (piece & 3);
                // the second panel's lanes store their halves the other way round: no two lanes of a row
                // on the same banks
                const bool swap = (piece >> 2) != 0;
                *reinterpret_cast<uint4*>(dst + kk * 128 + (((swap ? c + 1 : c) ^ (kk & 7)) << 4)) = swap ? hi4 : lo4;
                *reinterpret_cast<uint4*>(dst + kk * 128 + (((swap ? c : c + 1) ^ (kk & 7)) << 4)) = swap ? lo4 : hi4;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                t5_bar_arrive(t5_smem(full + n % S::RING));
                t5_bar_arrive(t5_smem(raw_empty + n % S::RAW_RING));
            }
        };
        // The first of these warps brings the scales: lane 8 u + i block i of the keys (u = 0) or values
        // (u = 1), fetched a tile ahead, its page two tiles ahead.
        const int sblk = SB_KV8_BLOCK * (lane & 7);
        const uint16_t* const scales = (lane & 8) ? a.v_scale : a.k_scale;
        const bool brings = warp == 8 && lane < 2 * PR_BLOCKS;
        auto entry_of = [&](int j) -> int {
            const int key = k0 + j * PR_KEYS + sblk;
            return brings && key < k1 ? a.g.table[(int64_t)b * a.g.table_stride + key / a.g.page_tokens] : -1;
        };
        auto scale_of = [&](int j, int entry) -> uint16_t {
            if (entry < 0 || entry >= a.g.pages) return 0;
            const int slot = (k0 + j * PR_KEYS + sblk) % a.g.page_tokens;
            return scales[((int64_t)entry * a.g.heads + head) * (a.g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK];
        };
        uint16_t scale = scale_of(0, entry_of(0));
        int entry = entry_of(1);
        for (int n = 0; n < 2 * ntiles; ++n) {
            if (!wait(empty + n % S::RING, n / S::RING + 1)) break;
            if (warp == 8 && !(n & 1)) {
                // whoever read the scales of four tiles ago is done: the slot's last tile came after them
                const int j = n >> 1;
                if (brings) sc[16 * (j & 3) + lane] = __uint_as_float((uint32_t)scale << 16);
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(scfull + (j & 3)));
                scale = scale_of(j + 1, entry);
                entry = entry_of(j + 2);
            }
            if (!wait(raw_full + n % S::RAW_RING, n / S::RAW_RING)) break;
            convert(n);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_REST));
    }
    if (warp == 13) {
        // ---- copies: a tile is eight scale blocks, each contiguous in its page; lane i brings block i ----
        const unsigned bytes = (unsigned)(SB_KV8_BLOCK * D);
        auto entry_of = [&](int j) -> int {
            const int key = k0 + j * PR_KEYS + SB_KV8_BLOCK * lane;
            return lane < PR_BLOCKS && key < k1 ? a.g.table[(int64_t)b * a.g.table_stride + key / a.g.page_tokens] : -1;
        };
        int entry = entry_of(0), issued = 0;
        for (int n = 0; n < 2 * ntiles; n += 2) {
            const int j = n >> 1, key = k0 + j * PR_KEYS + SB_KV8_BLOCK * lane;
            const int slot = key % a.g.page_tokens;
            const bool inside = lane < PR_BLOCKS && key < k1, fine = inside && entry >= 0 && entry < a.g.pages;
            if (inside && !fine) sb_latch(a.st, SB_ERR_INVALID, SBK_KV8);
            const int64_t at = (((int64_t)entry * a.g.heads + head) * a.g.page_tokens + slot) * D;
            const unsigned count = (unsigned)__popc(__ballot_sync(0xffffffffu, fine));
            entry = entry_of(j + 1);
            bool ok = true;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int rs = (n + u) % S::RAW_RING;
                ok = ok && wait(raw_empty + rs, (n + u) / S::RAW_RING + 1);
                if (!ok) break;
                const unsigned bar = t5_smem(raw_full + rs);
                if (lane == 0) t5_bar_expect(bar, count * bytes);
                __syncwarp();
                if (fine) t5_load_bulk(t5_smem(smem + S::RAW_AT + rs * S::RAW) + (unsigned)lane * bytes, (u ? a.v : a.k) + at, bytes, bar);
                __syncwarp();
                ++issued;
            }
            if (!ok) break;
        }
        // copies in flight land before the block leaves
        for (int i = max(0, issued - S::RAW_RING); i < issued; ++i)
            t5_bar_drain(t5_smem(raw_full + i % S::RAW_RING), (unsigned)(i / S::RAW_RING) & 1u);
    } else if (warp == 12 || (warp == 14 && two)) {
        // ---- products of one row tile ----
        const int qt = warp == 14;
        const bool one = t5_elect();
        // n: half of a key tile
        auto scores = [&](int n) {
            const unsigned q = t5_smem(smem + S::Q_AT + qt * S::OPERAND);
            const unsigned k = t5_smem(smem + S::T_AT + (n & ~1) % S::RING * S::OPERAND) + (unsigned)((n & 1) * PR_SUB * 128);
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
                pr_mma_ss(one, tmem + S::S_COL + qt * 128 + (n & 1) * PR_SUB, t5_desc_sw128(q + (s >> 2) * S::PANEL + 32 * (s & 3)),
                          t5_desc_sw128(k + (s >> 2) * S::PANEL + 32 * (s & 3)), pr_idesc(PR_SUB, false), s > 0);
            pr_commit(one, t5_smem(sfull + 2 * qt + (n & 1)));
        };
        auto values = [&](int n) {
            const unsigned v = t5_smem(smem + S::T_AT + (n | 1) % S::RING * S::OPERAND) + (unsigned)((n & 1) * PR_SUB * 128);
#pragma unroll
            for (int s = 0; s < PR_SUB / 16; ++s)
                pr_mma_ts(one, tmem + S::O_COL + qt * DP, tmem + S::S_COL + qt * 128 + (n & 1) * PR_SUB + 8 * s, pr_desc_v<DP>(v + 2048 * s),
                          pr_idesc(DP, true), n > 0 || s > 0);
            pr_commit(one, t5_smem(odone + qt));
        };
        // converted tiles in the order K 0, V 0, K 1, V 1, ...: the halves 2 j and 2 j + 1 use tiles
        // 2 j (keys) and 2 j + 1 (values)
        auto there = [&](int tile) { return wait(full + tile % S::RING, tile / S::RING); };
        auto done = [&](int tile) { pr_commit(one, t5_smem(empty + tile % S::RING)); };
        const int halves = 2 * ntiles;
        bool ok = wait(qready + qt, 0) && there(0);
        if (ok) {
            t5_fence_after();
            scores(0);
            scores(1);
            done(0);
        }
        for (int n = 0; ok && n < halves; ++n) {
            const int tile = n & ~1;
            ok = ((n & 1) || there(tile + 1)) && wait(pfull + 2 * qt + (n & 1), n >> 1);
            if (!ok) break;
            t5_fence_after();
            values(n);
            if (n & 1) done(tile + 1);
            if (n + 2 < halves) {
                // The same half of the next tile's scores, into the columns the weights were read from.
                // Products of different shapes are not ordered by their issue: those have to be done.
                ok = ((n & 1) || there(tile + 2)) && wait(odone + qt, n);
                if (!ok) break;
                t5_fence_after();
                scores(n + 2);
                if (n & 1) done(tile + 2);
            }
        }
        if (!ok) {                                   // what was issued still reads shared memory
            pr_commit(one, t5_smem(last + qt));
            t5_bar_drain(t5_smem(last + qt), 0u);
        }
    }
    __syncwarp();
    t5_fence_before();
    __syncthreads();
    if (warp == 12) {
        t5_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
    }
    if (threadIdx.x == 0 && *abort_flag) sb_latch(a.st, SB_ERR_TIMEOUT, SBK_KV8);
}

// the chunks of a row, in their order
__global__ void __launch_bounds__(128)
kv8_prompt_sum_kernel(const AtArgs a) {
    const int b = blockIdx.z, head = blockIdx.y;
    Kv8Request rq;
    if (!kv8_request(a.g, b, rq, a.st)) return;
    const int rows = rq.n * a.group, D = a.g.dim, quads = D / 4;
    const int64_t unit = (int64_t)blockIdx.x * 128 + threadIdx.x;
    const int row = (int)(unit / quads), d = 4 * (int)(unit - (int64_t)row * quads);
    if (row >= rows) return;
    const int rt = row / (2 * PR_ROWS), r = row % (2 * PR_ROWS);
    const int64_t at = (((int64_t)b * a.g.heads + head) * a.row_tiles + rt) * a.splits * (2 * PR_ROWS) + r;
    float m = -INFINITY, l = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x = 0; x < a.splits; ++x) {
        const float2 ml = a.part_ml[at + (int64_t)x * (2 * PR_ROWS)];
        if (ml.x == -INFINITY) continue;
        const float4 y = *reinterpret_cast<const float4*>(a.part + (at + (int64_t)x * (2 * PR_ROWS)) * D + d);
        const float mn = fmaxf(m, ml.x);
        const float f = m == -INFINITY ? 0.f : at_exp2(m - mn), h = at_exp2(ml.x - mn);
        l = fmaf(l, f, ml.y * h);
        v.x = fmaf(v.x, f, y.x * h); v.y = fmaf(v.y, f, y.y * h); v.z = fmaf(v.z, f, y.z * h); v.w = fmaf(v.w, f, y.w * h);
        m = mn;
    }
    const int64_t tok = rq.row0 + row / a.group;
    const int h = head * a.group + row % a.group;
    const float f = at_norm(l);
    *reinterpret_cast<uint2*>(a.o + tok * a.o_token_stride + h * a.o_head_stride + d) =
        make_uint2(u32(__floats2bfloat162_rn(v.x * f, v.y * f)), u32(__floats2bfloat162_rn(v.z * f, v.w * f)));
    if (d == 0 && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(m, l);
}

template <int TYPE, int DP>
sb_status prompt_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = PrShape<DP>;
    auto* kernel = kv8_prompt_kernel<TYPE, DP>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (max_new * a.group + 2 * PR_ROWS - 1) / (2 * PR_ROWS);
    int64_t keys = max_len;
    if (a.window > 0 && keys > a.window + max_new + PR_KEYS) keys = a.window + max_new + PR_KEYS;
    const int64_t tiles = row_tiles * a.g.heads * a.g.requests;
    // with fewer tiles than SMs the keys are cut too, into chunks of at least 8 tiles
    int64_t splits = tiles < ctx->sm_count ? ctx->sm_count / tiles : 1;
    if (splits > (keys + 8 * PR_KEYS - 1) / (8 * PR_KEYS)) splits = (keys + 8 * PR_KEYS - 1) / (8 * PR_KEYS);
    if (splits < 1) splits = 1;
    a.chunk = (int)(((keys + splits - 1) / splits + PR_KEYS - 1) / PR_KEYS * PR_KEYS);
    a.splits = (int)((keys + a.chunk - 1) / a.chunk);
    a.row_tiles = (int)row_tiles;
    if (row_tiles * a.splits > 65535) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: too many query rows");
    if (a.splits > 1) {
        const size_t n = (size_t)tiles * a.splits * (2 * PR_ROWS);
        void* arena;
        const sb_status s = sb_scratch(ctx, Carver::need({n * a.g.dim * 4, n * 8}), &arena);
        if (s != SB_OK) return s;
        Carver cv(arena);
        a.part = cv.take<float>(n * a.g.dim);
        a.part_ml = cv.take<float2>(n);
    }
    const dim3 grid((unsigned)a.g.heads, (unsigned)(row_tiles * a.splits), (unsigned)a.g.requests);
    kernel<<<grid, PR_THREADS, S::SMEM, ctx->stream>>>(a);
    SB_LAUNCHED(ctx);
    if (a.splits > 1) {
        const int64_t blocks = (max_new * a.group * (a.g.dim / 4) + 127) / 128;
        kv8_prompt_sum_kernel<<<dim3((unsigned)blocks, (unsigned)a.g.heads, (unsigned)a.g.requests), 128, 0, ctx->stream>>>(a);
        SB_LAUNCHED(ctx);
    }
    return SB_OK;
}

}  // namespace

sb_status kv8_prompt(sb_ctx* ctx, AtArgs a, int type, int64_t max_new, int64_t max_len) {
    if (type == SB_KV_INT8)
        return a.g.dim <= 64 ? prompt_launch<SB_KV_INT8, 64>(ctx, a, max_new, max_len) : prompt_launch<SB_KV_INT8, 128>(ctx, a, max_new, max_len);
    return a.g.dim <= 64 ? prompt_launch<SB_KV_E4M3, 64>(ctx, a, max_new, max_len) : prompt_launch<SB_KV_E4M3, 128>(ctx, a, max_new, max_len);
}
