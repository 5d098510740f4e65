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
// maximum of a row is only moved when it is off by more than 2^8 (with value scales P stays below 2^15, inside
// fp16), so sums in tensor memory are rarely touched between tiles.
//
// A step first takes the weights by the reference there is and looks at their sum: where that is small no
// maximum is needed (287 -> 273 us in the case below). The work is cut into equal shares (see
// kv8_attention.cuh); a sum kernel adds the pieces of items that several shares hold.
//
// What bounds it: per 128 keys of 256 rows the products need 2560 cycles (the scores, both operands from
// shared memory in halves of 64 keys, 1536 of them) and the exponentials 2048 (16 per cycle and SM); the kernel
// takes 4400, because a row tile's scores, softmax, weights, sums and next scores wait for one
// another. Half tiles and two row tiles overlap these chains; whole tiles per step were slower (339 us against
// 287), and so was a warp of its own for the scores (344).
// 4 requests of up to 1024 tokens behind up to 8192, 32 query heads of 128 over 8, e4m3: 255 us,
// 761 TFLOP/s, tensor pipe 54 % active; heads of 64 231 us, of 80 and 96 252.
#include "kv8_attention.cuh"
#include "tensor5.cuh"

namespace {

constexpr int PR_ROWS = 128;             // query rows of a tile; two per CTA
constexpr int PR_KEYS = 128;             // keys of a tile
constexpr int PR_BLOCKS = PR_KEYS / SB_KV8_BLOCK;
constexpr int PR_SUB = 64;               // keys of a softmax step: half a tile
constexpr int PR_SUBBLOCKS = PR_SUB / SB_KV8_BLOCK;
constexpr int PR_THREADS = 16 * 32;       // warp 15 only lends its registers
// Registers: the split at which nothing spills. 160/96/96 spilled 256 bytes a thread and took 273 us where this one
// takes 255; no split at all (128 each) 265.
// A softmax, conversion and other warp's thread: 8 x 136 + 4 x 120 + 4 x 120 warps' shares <= 16 x 128
constexpr int PR_REGS_SOFTMAX = 136, PR_REGS_CONVERT = 120, PR_REGS_REST = 120;
static_assert(8 * PR_REGS_SOFTMAX + 4 * PR_REGS_CONVERT + 4 * PR_REGS_REST <= 16 * 128, "what the block was launched with");
constexpr int PR_EXTRA = 6;              // what an item costs besides its key tiles, in key tiles: 14 us to 2.5 us a tile;
                                         // 4, 6 and 8 took 272, 262 and 267 us
constexpr int PR_LEAST = 4;              // units of a share at least: one request of 332 tokens took 34 us with 7, 30 with 4;
                                         // 30 tokens in 9000 38 and 41
constexpr float PR_LIMIT = 256.f;        // 2^AT_SLACK: largest sum of a half tile's weights before the row's reference moves

template <int DP>
struct PrShape {
    static constexpr int PANELS = DP / 64;                          // 128-byte columns of an operand row
    static constexpr int PANEL = 128 * 128;                         // bytes: 128 rows x 128
    static constexpr int OPERAND = PANELS * PANEL;
    static constexpr int RING = 3, RAW_RING = 4;                    // converted and raw tiles: K, V, K, V, ...
    static constexpr int RAW = PR_KEYS * DP;
    static constexpr int Q_AT = 0, T_AT = 2 * OPERAND, RAW_AT = T_AT + RING * OPERAND;
    static constexpr int SC_AT = RAW_AT + RAW_RING * RAW;           // scales of four tiles: 8 of K, 8 of V
    static constexpr int F_AT = SC_AT + 4 * 64;                      // score factor of a row, fp32
    static constexpr int BAR_AT = F_AT + 2 * PR_ROWS * 4;
    static constexpr int SMEM = BAR_AT + 304 + 1024;
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
// Largest score of a row and of each 16 columns, in units of log2 (kf: their factors, not negative).
__device__ __forceinline__ float pr_max(unsigned (&s)[PR_SUB / 32][32], const float (&kf)[PR_SUBBLOCKS], int upto, int from,
                                        float (&tops)[PR_SUBBLOCKS]) {
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
                if (c > upto || c <= from) x[u] = -INFINITY;
            }
            bm[0] = fmaxf(fmaxf(bm[0], x[0]), x[1]);
            bm[1] = fmaxf(fmaxf(bm[1], x[2]), x[3]);
        }
        const float top = fmaxf(bm[0], bm[1]);
        // a factor of 0 makes 0 of any score, but no NaN of a block that is masked whole
        tops[h] = top == -INFINITY ? -INFINITY : top * kf[h];
        mx = fmaxf(mx, tops[h]);
    }
    return mx;
}
// The row's weights 2^(score - ref), times the value scale of their 16 columns, in fp16 over the
// scores; returns the sum of the weights.
template <bool EDGE>
__device__ __forceinline__ float pr_weights(unsigned ts, unsigned (&s)[PR_SUB / 32][32], const float (&kf)[PR_SUBBLOCKS],
                                            const float (&vw)[PR_SUBBLOCKS], float ref, int upto, int from) {
    f32x2 sum[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
    const f32x2 off = pk2(-ref, -ref);
#pragma unroll
    for (int c = 0; c < PR_SUB / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x2 w = pk2(vw[2 * c + h], vw[2 * c + h]), kk = pk2(kf[2 * c + h], kf[2 * c + h]);
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float e[2];
                upk2(fma2(pk2(__uint_as_float(s[c][16 * h + i]), __uint_as_float(s[c][16 * h + i + 1])), kk, off), e[0], e[1]);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    e[u] = at_exp2(e[u]);
                    if (EDGE && (32 * c + 16 * h + i + u > upto || 32 * c + 16 * h + i + u <= from)) e[u] = 0.f;
                }
                const f32x2 x = pk2(e[0], e[1]);
                sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], x);
                upk2(mul2(x, w), e[0], e[1]);
                p[8 * h + i / 2] = at_half2(e[0], e[1]);
            }
        }
        pr_st16(ts + 16 * c, p);
    }
    float lo, hi;
    upk2(add2(sum[0], sum[1]), lo, hi);
    return lo + hi;
}

// The plan of the shares (items: 256 query rows), written by a kernel of its own.
struct PrWork {
    long long* prefix;           // [row tiles of all requests + 1] units of one head before the row tile
    int4* start;                 // [ctas] (row tile of all requests, head, unit) a share starts with; x < 0: no share
    long long* share;            // units of a share; units in all
    int ctas;
};
using PrWalk = AtWalk<2 * PR_ROWS, PR_KEYS, PR_EXTRA>;
__device__ __forceinline__ int pr_units(const AtArgs& a, int row_tile) {
    const int steps = at_item<2 * PR_ROWS, PR_KEYS>(a, row_tile).steps;
    return steps ? steps + PR_EXTRA : 0;
}
__global__ void __launch_bounds__(1024)
kv8_prompt_plan_kernel(const AtArgs a, const PrWork w) {
    __shared__ long long warp_sum_at[32], total_at;
    const int n = a.row_tiles * a.g.requests, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    at_let_next();
    long long before = 0;
    for (int base = 0; base < n; base += 1024) {
        const int i = base + threadIdx.x;
        const long long mine = i < n ? pr_units(a, i) : 0;
        long long x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sum_at[warp] = x;
        __syncthreads();
        if (warp == 0) {
            long long t = warp_sum_at[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, t, o);
                if (lane >= o) t += y;
            }
            warp_sum_at[lane] = t;
            if (lane == 31) total_at = t;
        }
        __syncthreads();
        if (i < n) w.prefix[i] = before + x - mine + (warp ? warp_sum_at[warp - 1] : 0);
        before += total_at;
        __syncthreads();
    }
    if (threadIdx.x == 0) w.prefix[n] = before;
    __syncthreads();
    const long long total = before * a.g.heads;
    const long long share = max((total + w.ctas - 1) / w.ctas, (long long)PR_LEAST);
    if (threadIdx.x == 0) { w.share[0] = share; w.share[1] = total; }
    for (int c = threadIdx.x; c < w.ctas; c += 1024) {
        const long long at = c * share;
        if (at >= total) { w.start[c] = make_int4(-1, 0, 0, 0); continue; }
        int lo = 0, hi = n;                                          // the last row tile that starts at or before `at`
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (w.prefix[mid] * a.g.heads <= at) lo = mid; else hi = mid;
        }
        const long long rest = at - w.prefix[lo] * a.g.heads, units = w.prefix[lo + 1] - w.prefix[lo];
        w.start[c] = make_int4(lo, (int)(rest / units), (int)(rest % units), 0);
    }
}

template <int TYPE, int DP>
__global__ void __launch_bounds__(PR_THREADS, 1)
kv8_prompt_kernel(const AtArgs a, const PrWork work) {
    using S = PrShape<DP>;
    extern __shared__ unsigned char pr_raw[];
    unsigned char* smem = pr_raw + ((1024u - (t5_smem(pr_raw) & 1023u)) & 1023u);
    float* sc = reinterpret_cast<float*>(smem + S::SC_AT);           // [4][16]
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + S::BAR_AT);
    // raw tiles: landed, converted; converted tiles: there, multiplied; per row tile (and half of a key
    // tile): scores, weights, sums; all sums of a piece.  A wait tells a phase from its neighbours only
    // (one bit), so every barrier is waited for by someone who cannot be two phases away: the next phases wait for
    // something he does later, and what he has waited for before holds the phase before to have ended.
    unsigned long long *raw_full = bars, *raw_empty = bars + 4, *full = bars + 8, *empty = bars + 12, *sfull = bars + 16,
                       *pfull = bars + 20, *odone = bars + 24, *scfull = bars + 26, *qready = bars + 30, *last = bars + 32, *fin = bars + 34;
    unsigned* tmem_slot = reinterpret_cast<unsigned*>(bars + 36);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int D = a.g.dim;
    PrWalk wk;
    at_after_previous();
    at_let_next();                           // its blocks find room when these end, and wait for that
    {
        const int4 s = work.start[blockIdx.x];
        const long long share = work.share[0], at = blockIdx.x * share;
        if (s.x < 0 || !wk.begin(a, s.x, s.y, s.z, at, min(share, work.share[1] - at))) return;
    }

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::RAW_RING; ++i) {
            t5_bar_init(t5_smem(raw_full + i), 1);
            t5_bar_init(t5_smem(raw_empty + i), 4);
        }
        for (int i = 0; i < S::RING; ++i) {
            t5_bar_init(t5_smem(full + i), 4);
            t5_bar_init(t5_smem(empty + i), 2);
        }
        for (int i = 0; i < 4; ++i) {
            t5_bar_init(t5_smem(sfull + i), 1);
            t5_bar_init(t5_smem(pfull + i), 4);
            t5_bar_init(t5_smem(scfull + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            t5_bar_init(t5_smem(odone + i), 1);
            t5_bar_init(t5_smem(qready + i), 4);
            t5_bar_init(t5_smem(last + i), 1);
            t5_bar_init(t5_smem(fin + i), 1);
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
        const unsigned lanes = (unsigned)((warp & 3) * 32) << 16;
        const unsigned ts = tmem + lanes + S::S_COL + qt * 128, to = tmem + lanes + S::O_COL + qt * DP;
        int tiles_all = 0, tiles_mine = 0, pieces = 0;               // key tiles and pieces so far (of this row tile)
        bool ok = true, skipped = false;
        for (bool more = true; more && ok; more = wk.next(a), ++tiles_all) {
            const AtItem& it = wk.it;
            const int count = wk.count;
            tiles_all += count - 1;
            const int base_all = tiles_all - (count - 1);
            // No rows: nothing of these tiles waits for these warps, so they must not wait for a phase of them either (two
            // phases late they would wait for one that may never come).
            if (it.nrow <= qt * PR_ROWS) {
                skipped = true;
                continue;
            }
            const int r = threadIdx.x, row = it.r0 + r;              // row of the item, of the request
            const bool real = r < it.nrow;
            {
                // rows by half warps, 16 bytes a lane: the largest element, the scaling, fp16 into the
                // swizzled operand
                constexpr int LANES = DP / 8, RPI = 32 / LANES, NI = 32 / RPI;      // lanes of a row, rows at a time
                const int c = lane % LANES, sub = lane / LANES;
                float* factor = reinterpret_cast<float*>(smem + S::F_AT) + qt * PR_ROWS;
                unsigned char* q0 = smem + S::Q_AT + qt * S::OPERAND + (c >> 3) * S::PANEL;
                const int tok0 = a.by_group.quot(it.r0), head0 = it.r0 - tok0 * a.group;
                const __nv_bfloat16* src = a.q + (int64_t)(it.rq.row0 + tok0) * a.q_token_stride + (int64_t)wk.head * a.group * a.q_head_stride + 8 * c;
                uint4 x[NI];
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int rr = qt * PR_ROWS + (warp & 3) * 32 + i * RPI + sub, at = head0 + rr;
                    const int tok = a.by_group.quot(at);
                    x[i] = make_uint4(0, 0, 0, 0);
                    if (rr < it.nrow && 8 * c < D)
                        x[i] = *reinterpret_cast<const uint4*>(src + tok * a.q_token_stride + (at - tok * a.group) * a.q_head_stride);
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    uint32_t m = __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
#pragma unroll
                    for (int o = 1; o < LANES; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                    const float up = at_query_scale(max(m & 0xffffu, m >> 16)), by = at_signed(up, a.scale_log2);
                    const int rr = (warp & 3) * 32 + i * RPI + sub;
                    if (c == 0) factor[rr] = up;
                    *reinterpret_cast<uint4*>(q0 + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) =
                        make_uint4(at_half2(bf16lo(x[i].x) * by, bf16hi(x[i].x) * by), at_half2(bf16lo(x[i].y) * by, bf16hi(x[i].y) * by),
                                   at_half2(bf16lo(x[i].z) * by, bf16hi(x[i].z) * by), at_half2(bf16lo(x[i].w) * by, bf16hi(x[i].w) * by));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(qready + qt));
            }
            const float fq = __fdiv_rn(fabsf(a.scale_log2), reinterpret_cast<const float*>(smem + S::F_AT)[r]);
            // (a thread without a row has queries of zeros, and its results go nowhere)
            const int pos = it.rq.past + a.by_group.quot(row);
            // positions of the tile's first and last row decide which key tiles need a mask
            const int pos_lo = it.rq.past + a.by_group.quot(it.r0 + qt * PR_ROWS);
            const int pos_hi = it.rq.past + a.by_group.quot(it.r0 + min(it.nrow, (qt + 1) * PR_ROWS) - 1);
            const int k0 = it.lo + wk.step0 * PR_KEYS, k1 = min(it.hi, k0 + count * PR_KEYS);
            float m = -INFINITY, l = 0.f, inv = 0.f;
            // After tiles without rows the scales' phase before this one need not have ended. It has once there are scores: a
            // tile's scales come before its keys are converted.
            if (skipped) ok = wait(sfull + 2 * qt, tiles_mine);
            skipped = false;
            ok = ok && wait(scfull + (base_all & 3), base_all >> 2);
            for (int n = 0; ok && n < 2 * count; ++n) {              // halves of the key tiles
                const int j = n >> 1, u = n & 1;
                ok = wait(sfull + 2 * qt + u, tiles_mine + j);
                if (!ok) break;
                t5_fence_after();
                unsigned s[PR_SUB / 32][32];
                t5_ld32(ts + PR_SUB * u, s[0]);
                t5_ld32(ts + PR_SUB * u + 32, s[1]);
                const int key = k0 + n * PR_SUB;
                const bool edge = key + PR_SUB > pos_lo + 1 || key + PR_SUB > k1 || (a.window > 0 && key <= pos_hi - a.window);
                const float4* scj = reinterpret_cast<const float4*>(sc + 16 * ((base_all + j) & 3) + PR_SUBBLOCKS * u);
                const float4 k4 = scj[0], v4 = scj[PR_BLOCKS / 4];
                const float kf[PR_SUBBLOCKS] = {k4.x * fq, k4.y * fq, k4.z * fq, k4.w * fq};
                const float vmax = fmaxf(fmaxf(v4.x, v4.y), fmaxf(v4.z, v4.w));
                const int upto = min(pos, k1 - 1) - key, from = a.window > 0 ? pos - a.window - key : -1;
                // Where nothing is masked, the weights by the reference there is; their sum says whether it
                // still does: no weight is above their sum. One above PR_LIMIT (or none: NaN), a mask, a
                // first key or a value scale too large takes the other way, by the row's maximum.
                float sum = 0.f;
                bool again = edge || __any_sync(0xffffffffu, m == -INFINITY || vmax * inv > AT_TOP);
                t5_wait_ld();
                if (!again) {
                    const float vw[PR_SUBBLOCKS] = {v4.x * inv, v4.y * inv, v4.z * inv, v4.w * inv};
                    sum = pr_weights<false>(ts + PR_SUB * u, s, kf, vw, m, upto, from);
                    again = __any_sync(0xffffffffu, !(sum <= PR_LIMIT));
                }
                if (again) {
                    float tops[PR_SUBBLOCKS];
                    const float mx = pr_max(s, kf, upto, from, tops);
                    const bool far = mx > m + AT_SLACK || (m == -INFINITY && mx > m) || vmax * inv > AT_TOP;
                    float f = 1.f;
                    if (far) {
                        const float ref = fmaxf(m, mx), down = m == -INFINITY ? 0.f : at_exp2(m - ref), held = at_power_inv(inv) * down;
                        const float most = fmaxf(fmaxf(at_exp2(tops[0] - ref) * v4.x, at_exp2(tops[1] - ref) * v4.y),
                                                 fmaxf(at_exp2(tops[2] - ref) * v4.z, at_exp2(tops[3] - ref) * v4.w));
                        inv = at_value_inv(most, held, vmax);
                        m = ref;
                        l *= down;
                        f = held * inv;
                    }
                    if (__any_sync(0xffffffffu, far) && n > 0) {
                        // the sums so far: the products of the half before this one have to be done
                        ok = wait(odone + qt, 2 * tiles_mine + n - 1);
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
                    const float ref = m == -INFINITY ? 0.f : m;
                    const float vw[PR_SUBBLOCKS] = {v4.x * inv, v4.y * inv, v4.z * inv, v4.w * inv};
                    pr_wait_st();
                    sum = pr_weights<true>(ts + PR_SUB * u, s, kf, vw, ref, upto, from);
                }
                l += sum;
                pr_wait_st();
                t5_fence_before();
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(pfull + 2 * qt + u));
                if (u && j + 1 < count) ok = wait(scfull + ((base_all + j + 1) & 3), (base_all + j + 1) >> 2);
            }
            // ---- results ----
            if (ok) ok = wait(fin + qt, pieces);
            if (!ok) break;
            t5_fence_after();
            tiles_mine += count;
            ++pieces;
            const bool whole = count == it.steps;
            const int h0 = wk.head * a.group;
            const int64_t tok = it.rq.row0 + a.by_group.quot(row);
            const int h = h0 + a.by_group.rem(row);
            const float back = at_power_inv(inv), norm = whole ? at_norm(l) * back : back;
            const int64_t slot = 2 * (int64_t)blockIdx.x + (wk.first ? 0 : 1);
            // this warp's rows in bf16 where its queries were, in the same order
            unsigned char* o0 = smem + S::Q_AT + qt * S::OPERAND + (warp & 3) * 32 * 128;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                unsigned o[32];
                t5_ld32(to + c, o);
                t5_wait_ld();
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (c + i < D)
                            *reinterpret_cast<float4*>(a.part + ((slot * (D / 4) + (c + i) / 4) * (2 * PR_ROWS) + r) * 4) =
                                make_float4(__uint_as_float(o[i]) * norm, __uint_as_float(o[i + 1]) * norm,
                                            __uint_as_float(o[i + 2]) * norm, __uint_as_float(o[i + 3]) * norm);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            w[u] = u32(__floats2bfloat162_rn(__uint_as_float(o[i + 2 * u]) * norm, __uint_as_float(o[i + 2 * u + 1]) * norm));
                        *reinterpret_cast<uint4*>(o0 + ((c + i) >> 6) * S::PANEL + lane * 128 + (((((c + i) >> 3) & 7) ^ (lane & 7)) << 4)) =
                            make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (whole) {
                __syncwarp();
                constexpr int LANES = DP / 8, RPI = 32 / LANES;
                const int c = lane % LANES, sub = lane / LANES;
                const int tok0 = a.by_group.quot(it.r0), head0 = it.r0 - tok0 * a.group;
                __nv_bfloat16* dst = a.o + (int64_t)(it.rq.row0 + tok0) * a.o_token_stride + (int64_t)h0 * a.o_head_stride + 8 * c;
#pragma unroll 4
                for (int i = 0; i < 32; i += RPI) {
                    const int rl = i + sub, rr = qt * PR_ROWS + (warp & 3) * 32 + rl, at = head0 + rr;
                    const int tk = a.by_group.quot(at);
                    const uint4 v = *reinterpret_cast<const uint4*>(o0 + (c >> 3) * S::PANEL + rl * 128 + (((c & 7) ^ (rl & 7)) << 4));
                    if (rr < it.nrow && 8 * c < D)
                        *reinterpret_cast<uint4*>(dst + tk * a.o_token_stride + (at - tk * a.group) * a.o_head_stride) = v;
                }
                __syncwarp();
                if (real && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(m, l);
            } else if (real) a.part_ml[slot * (2 * PR_ROWS) + r] = make_float2(m, l);
            t5_fence_before();                                       // the sums are read before the next piece's products
        }
    } else if (warp < 12) {
        // ---- conversion: a thread takes one 16-byte piece of every PASS-th row of a tile ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_CONVERT));
        constexpr int PIECES = DP / 16, PASS = 128 / PIECES, NP = PR_KEYS / PASS;
        const int tid = threadIdx.x - 256, piece = tid % PIECES, krow = tid / PIECES;
        // n: converted tile of all, left: rows that were copied and belong to the request (the rest: zeros)
        auto convert = [&](int n, int left) {
            const unsigned src = t5_smem(smem + S::RAW_AT + n % S::RAW_RING * S::RAW) + (unsigned)(krow * D + 16 * piece);
            unsigned char* dst = smem + S::T_AT + n % S::RING * S::OPERAND + (piece >> 2) * S::PANEL;
            if (16 * piece >= D) left = 0;
            uint4 x[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                x[i] = make_uint4(0, 0, 0, 0);
                if (krow + PASS * i < left) x[i] = at_lds128(src + (unsigned)(PASS * i * D));
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int kk = krow + PASS * i;
                // the second panel's lanes convert and store their halves the other way round: no two lanes
                // of a row on the same banks
                const bool swap = (piece >> 2) != 0;
                const int c = 2 * (piece & 3);
                const uint32_t w[4] = {at_flip<TYPE>(swap ? x[i].z : x[i].x), at_flip<TYPE>(swap ? x[i].w : x[i].y),
                                       at_flip<TYPE>(swap ? x[i].x : x[i].z), at_flip<TYPE>(swap ? x[i].y : x[i].w)};
                *reinterpret_cast<uint4*>(dst + kk * 128 + (((swap ? c + 1 : c) ^ (kk & 7)) << 4)) =
                    make_uint4(at_pair<TYPE, 0>(w[0]), at_pair<TYPE, 1>(w[0]), at_pair<TYPE, 0>(w[1]), at_pair<TYPE, 1>(w[1]));
                *reinterpret_cast<uint4*>(dst + kk * 128 + (((swap ? c : c + 1) ^ (kk & 7)) << 4)) =
                    make_uint4(at_pair<TYPE, 0>(w[2]), at_pair<TYPE, 1>(w[2]), at_pair<TYPE, 0>(w[3]), at_pair<TYPE, 1>(w[3]));
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
        bool ok = true;
        int n = 0;                                                   // converted tiles so far
        for (bool more = true; more && ok; more = wk.next(a)) {
            const int k0 = wk.it.lo + wk.step0 * PR_KEYS, k1 = min(wk.it.hi, k0 + wk.count * PR_KEYS);
            const int limit = min(wk.it.rq.len, (k1 + SB_KV8_BLOCK - 1) / SB_KV8_BLOCK * SB_KV8_BLOCK) - k0;
            auto entry_of = [&](int j) -> int {
                const int key = k0 + j * PR_KEYS + sblk;
                return brings && key < k1 ? a.g.table[(int64_t)wk.it.b * a.g.table_stride + a.g.page.quot(key)] : -1;
            };
            auto scale_of = [&](int j, int entry) -> uint16_t {
                if (entry < 0 || entry >= a.g.pages) return 0;
                const int slot = a.g.page.rem(k0 + j * PR_KEYS + sblk);
                return scales[((int64_t)entry * a.g.heads + wk.head) * (a.g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK];
            };
            uint16_t scale = scale_of(0, entry_of(0));
            int entry = entry_of(1);
            for (int i = 0; i < 2 * wk.count; ++i, ++n) {
                ok = wait(empty + n % S::RING, n / S::RING + 1);
                if (!ok) break;
                if (warp == 8 && !(i & 1)) {
                    // whoever read the scales of four tiles ago is done: the slot's last tile came after them
                    const int j = n >> 1;
                    if (brings) sc[16 * (j & 3) + lane] = __uint_as_float((uint32_t)scale << 16);
                    __syncwarp();
                    if (lane == 0) t5_bar_arrive(t5_smem(scfull + (j & 3)));
                    scale = scale_of((i >> 1) + 1, entry);
                    entry = entry_of((i >> 1) + 2);
                }
                ok = wait(raw_full + n % S::RAW_RING, n / S::RAW_RING);
                if (!ok) break;
                convert(n, limit - (i >> 1) * PR_KEYS);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_REST));
    }
    if (warp == 13) {
        // ---- copies: a tile is eight scale blocks, each contiguous in its page; lane i brings block i ----
        const unsigned bytes = (unsigned)(SB_KV8_BLOCK * D);
        bool ok = true;
        int issued = 0;
        for (bool more = true; more && ok; more = wk.next(a)) {
            const int k0 = wk.it.lo + wk.step0 * PR_KEYS, k1 = min(wk.it.hi, k0 + wk.count * PR_KEYS);
            auto entry_of = [&](int j) -> int {
                const int key = k0 + j * PR_KEYS + SB_KV8_BLOCK * lane;
                return lane < PR_BLOCKS && key < k1 ? a.g.table[(int64_t)wk.it.b * a.g.table_stride + a.g.page.quot(key)] : -1;
            };
            int entry = entry_of(0);
            for (int j = 0; ok && j < wk.count; ++j) {
                const int key = k0 + j * PR_KEYS + SB_KV8_BLOCK * lane;
                const int slot = a.g.page.rem(key);
                const bool inside = lane < PR_BLOCKS && key < k1, fine = inside && entry >= 0 && entry < a.g.pages;
                if (inside && !fine) sb_latch(a.st, SB_ERR_INVALID, SBK_KV8);
                const int64_t at = (((int64_t)entry * a.g.heads + wk.head) * a.g.page_tokens + slot) * D;
                const unsigned blocks = (unsigned)__popc(__ballot_sync(0xffffffffu, fine));
                entry = entry_of(j + 1);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int rs = issued % S::RAW_RING;
                    ok = ok && wait(raw_empty + rs, issued / S::RAW_RING + 1);
                    if (!ok) break;
                    const unsigned bar = t5_smem(raw_full + rs);
                    if (lane == 0) t5_bar_expect(bar, blocks * bytes);
                    __syncwarp();
                    if (fine) t5_load_bulk(t5_smem(smem + S::RAW_AT + rs * S::RAW) + (unsigned)lane * bytes, (u ? a.v : a.k) + at, bytes, bar);
                    __syncwarp();
                    ++issued;
                }
            }
        }
        // copies in flight land before the block leaves
        for (int i = max(0, issued - S::RAW_RING); i < issued; ++i)
            t5_bar_drain(t5_smem(raw_full + i % S::RAW_RING), (unsigned)(i / S::RAW_RING) & 1u);
    } else if (warp == 12 || warp == 14) {
        // ---- products of one row tile ----
        const int qt = warp == 14;
        const bool one = t5_elect();
        // h: half of a key tile, of all this row tile's; tile: converted tile of all
        auto scores = [&](int h, int tile) {
            const unsigned q = t5_smem(smem + S::Q_AT + qt * S::OPERAND);
            const unsigned k = t5_smem(smem + S::T_AT + tile % S::RING * S::OPERAND) + (unsigned)((h & 1) * PR_SUB * 128);
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
                pr_mma_ss(one, tmem + S::S_COL + qt * 128 + (h & 1) * PR_SUB, t5_desc_sw128(q + (s >> 2) * S::PANEL + 32 * (s & 3)),
                          t5_desc_sw128(k + (s >> 2) * S::PANEL + 32 * (s & 3)), pr_idesc(PR_SUB, false), s > 0);
            pr_commit(one, t5_smem(sfull + 2 * qt + (h & 1)));
        };
        auto values = [&](int h, int tile, bool add) {
            const unsigned v = t5_smem(smem + S::T_AT + tile % S::RING * S::OPERAND) + (unsigned)((h & 1) * PR_SUB * 128);
#pragma unroll
            for (int s = 0; s < PR_SUB / 16; ++s)
                pr_mma_ts(one, tmem + S::O_COL + qt * DP, tmem + S::S_COL + qt * 128 + (h & 1) * PR_SUB + 8 * s, pr_desc_v<DP>(v + 2048 * s),
                          pr_idesc(DP, true), add || s > 0);
            pr_commit(one, t5_smem(odone + qt));
        };
        auto there = [&](int tile) { return wait(full + tile % S::RING, tile / S::RING); };
        auto done = [&](int tile) { pr_commit(one, t5_smem(empty + tile % S::RING)); };
        bool ok = true;
        int t = 0, mine = 0, pieces = 0;                             // converted tiles (keys: even), this row tile's halves, pieces
        for (bool more = true; more && ok; more = wk.next(a)) {
            const int halves = 2 * wk.count;
            if (wk.it.nrow <= qt * PR_ROWS) {                        // no rows: lets the tiles go as they come
                for (int i = 0; ok && i < halves; ++i, ++t) {
                    ok = there(t);
                    if (ok) done(t);
                }
                continue;
            }
            ok = wait(qready + qt, pieces++) && there(t);
            if (ok) {
                t5_fence_after();
                scores(mine, t);
                scores(mine + 1, t);
                done(t);
            }
            for (int n = 0; ok && n < halves; ++n) {
                const int tile = t + (n & ~1);                       // this half's keys; its values: the next
                ok = ((n & 1) || there(tile + 1)) && wait(pfull + 2 * qt + (n & 1), (mine + n) >> 1);
                if (!ok) break;
                t5_fence_after();
                values(mine + n, tile + 1, n > 0);
                if (n & 1) done(tile + 1);
                if (n + 2 < halves) {
                    // The same half of the next tile's scores, into the columns the weights were read from.
                    // Products of different shapes are not ordered by their issue: those have to be done.
                    ok = ((n & 1) || there(tile + 2)) && wait(odone + qt, mine + n);
                    if (!ok) break;
                    t5_fence_after();
                    scores(mine + n + 2, tile + 2);
                    if (n & 1) done(tile + 2);
                }
            }
            if (ok) pr_commit(one, t5_smem(fin + qt));
            t += halves;
            mine += halves;
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

// The pieces of an item that lies in several shares, in their order. Block (c, y): the item that the
// border before share c + 1 cuts, if no earlier border does; 32 of its rows, eight threads a row, a
// thread every eighth four columns. The chain of dependent reads (share, item, sums) is what a block
// takes, so all columns go through it together (a block per 32 columns took 20 us for 4
// requests of up to 1024 tokens). What the plan says is read before the products have ended.
template <int DP>
__global__ void __launch_bounds__(256)
kv8_prompt_sum_kernel(const AtArgs a, const PrWork w) {
    constexpr int NQ = DP / 32;
    const int c = blockIdx.x + 1, D = a.g.dim;
    const int4 s = w.start[c];
    const long long share = w.share[0], from = c * share - s.z;      // the item's first unit of all
    // a border that lies before the first tile, or behind one that cuts the same item, has nothing to add
    bool mine = s.x >= 0 && s.z > PR_EXTRA;
    const int c0 = mine ? (int)((from + PR_EXTRA) / share) : 0;      // the share with its first tile
    mine = mine && c == c0 + 1;
    AtItem it{};
    if (mine) it = at_item<2 * PR_ROWS, PR_KEYS>(a, s.x);
    const int r = 32 * blockIdx.y + threadIdx.x / 8, quad0 = threadIdx.x % 8;
    at_after_previous();
    if (!mine || r >= it.nrow) return;
    const int c1 = (int)((from + it.steps + PR_EXTRA - 1) / share);
    float m = -INFINITY, l = 0.f;
    float4 v[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x = c0; x <= c1; ++x) {
        // the first piece of that share, unless the item starts inside the share
        const int64_t slot = 2 * (int64_t)x + (from > x * share ? 1 : 0);
        const float2 ml = a.part_ml[slot * (2 * PR_ROWS) + r];
        float4 y[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (4 * (quad0 + 8 * q) < D)
                y[q] = *reinterpret_cast<const float4*>(a.part + ((slot * (D / 4) + quad0 + 8 * q) * (2 * PR_ROWS) + r) * 4);
        }
        const float mn = fmaxf(m, ml.x);
        const float f = m == -INFINITY ? 0.f : at_exp2(m - mn), h = ml.x == -INFINITY ? 0.f : at_exp2(ml.x - mn);
        l = fmaf(l, f, ml.y * h);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            v[q].x = fmaf(v[q].x, f, y[q].x * h); v[q].y = fmaf(v[q].y, f, y[q].y * h);
            v[q].z = fmaf(v[q].z, f, y[q].z * h); v[q].w = fmaf(v[q].w, f, y[q].w * h);
        }
        m = mn;
    }
    const int row = it.r0 + r;
    const int64_t tok = it.rq.row0 + a.by_group.quot(row);
    const int h = s.y * a.group + a.by_group.rem(row);
    const float f = at_norm(l);
#pragma unroll
    for (int q = 0; q < NQ; ++q)
        if (4 * (quad0 + 8 * q) < D)
            *reinterpret_cast<uint2*>(a.o + tok * a.o_token_stride + h * a.o_head_stride + 4 * (quad0 + 8 * q)) =
                make_uint2(u32(__floats2bfloat162_rn(v[q].x * f, v[q].y * f)), u32(__floats2bfloat162_rn(v[q].z * f, v[q].w * f)));
    if (quad0 == 0 && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(m, l);
}

template <int TYPE, int DP>
sb_status prompt_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = PrShape<DP>;
    auto* kernel = kv8_prompt_kernel<TYPE, DP>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (max_new * a.group + 2 * PR_ROWS - 1) / (2 * PR_ROWS), n = row_tiles * a.g.requests;
    if (n >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: too many query rows");
    int64_t keys = max_len;
    if (a.window > 0 && keys > a.window + max_new + PR_KEYS) keys = a.window + max_new + PR_KEYS;
    // one share per SM, fewer if there cannot be so many shares
    const int64_t most = (n * a.g.heads * ((keys + PR_KEYS - 1) / PR_KEYS + 1 + PR_EXTRA) + PR_LEAST - 1) / PR_LEAST;
    PrWork w{};
    w.ctas = (int)(most < ctx->sm_count ? most : ctx->sm_count);
    a.row_tiles = (int)row_tiles;
    a.by_row_tiles = KvDiv(a.row_tiles);
    const size_t rows = (size_t)w.ctas * 2 * (2 * PR_ROWS);
    void* arena;
    const sb_status s = sb_scratch(ctx, Carver::need({((size_t)n + 1) * 8, (size_t)w.ctas * 16, 16, rows * a.g.dim * 4, rows * 8}), &arena);
    if (s != SB_OK) return s;
    Carver cv(arena);
    w.prefix = cv.take<long long>((size_t)n + 1);
    w.start = cv.take<int4>(w.ctas);
    w.share = cv.take<long long>(2);
    a.part = cv.take<float>(rows * a.g.dim);
    a.part_ml = cv.take<float2>(rows);
    kv8_prompt_plan_kernel<<<1, 1024, 0, ctx->stream>>>(a, w);
    SB_LAUNCHED(ctx);
    // The other two are sent off while the kernel before them still runs and wait on the device for its
    // end (at_after_previous), which hides their launches.
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.stream = ctx->stream;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)w.ctas);
    cfg.blockDim = dim3(PR_THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, a, w));
    SB_LAUNCHED(ctx);
    if (w.ctas > 1) {
        cfg.gridDim = dim3((unsigned)(w.ctas - 1), 2 * PR_ROWS / 32);
        cfg.blockDim = dim3(256);
        cfg.dynamicSmemBytes = 0;
        SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kv8_prompt_sum_kernel<DP>, a, w));
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
