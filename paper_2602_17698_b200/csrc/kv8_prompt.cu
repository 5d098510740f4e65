// Attention of many query rows over the 8-bit or the 4-bit cache (prompts and chunks of prompts) on tcgen05.
//
// A CTA takes 256 query rows of one cache head (new tokens x query heads that share it) as two
// tiles of 128, one row per softmax thread, and walks over the keys in tiles of 128:
//     S = Q K^T   (128 x 128, fp16 x fp16 -> fp32 in tensor memory)
//     P = 2^(S factor - m), times the value scale of its 16 keys, to fp16, over S's own columns
//     O += P V    (A from tensor memory, V with d contiguous, fp32 in tensor memory)
// The tensor cores cannot multiply 8-bit by 16-bit operands, so four warps convert a tile of K and
// of V to fp16 (exact) into the 128-byte-swizzled layout the instructions read; 256 rows share the
// conversion. Scales of the 8-bit cache never touch K and V: a scale block is 16 columns of S, its key scale goes
// into the factor of S, its value scale into P. A scale of the 4-bit cache belongs to 16 elements of one token: it is multiplied in
// when they are converted (exact in fp16), the heads' scales go into the factor of S and the results.
//
// Warps 0-3 and 4-7: softmax of the two tiles; 8-11: conversion; 12 and 14: their products; 13: copies. A softmax
// step takes half a key tile (64 keys): while it works on one half, the tensor cores multiply the
// other half's weights and put the next tile's scores in their place. The running
// maximum of a row is only moved when it is off by more than 2^8 (with value scales P stays below 2^15, inside
// fp16), so sums in tensor memory are rarely touched between tiles.
//
// A step first takes the weights by the reference there is and looks at their sum: where that is small no
// maximum is needed (287 -> 273 us in the case below). The work is cut into equal shares (see
// kv8_attention.cuh); a sum kernel adds the pieces of items that several shares hold. Short items have a CTA each (pr_direct).
//
// What bounds it: per 128 keys of 256 rows the products need 2560 cycles (the scores, both operands from
// shared memory in halves of 64 keys, 1536 of them) and the exponentials 2048 (16 per cycle and SM); the kernel
// takes 4400, because a row tile's scores, softmax, weights, sums and next scores wait for one
// another. Half tiles and two row tiles overlap these chains; whole tiles per step were slower (339 us against
// 287), and so was a warp of its own for the scores (344).
// 4 requests of up to 1024 tokens behind up to 8192, 32 query heads of 128 over 8, e4m3: 250 us,
// 776 TFLOP/s, tensor pipe 54 % active; heads of 64 231 us, of 80 and 96 252. Over the 4-bit cache 231 us, 841 TFLOP/s: half the bytes
// to copy, and no value scales in the softmax. 4 of up to 1024 behind 4096 with heads of 256 (one row tile, so every key tile is
// converted for 128 rows only): 0.88 ms, a third of the products' rate.
#include "kv8_attention.cuh"
#include "kv4.cuh"
#include "launch.cuh"
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
constexpr float PR_LIMIT4 = 16384.f;     // and over the 4-bit cache: 2^AT4_FAR
constexpr float PR_LIMIT = 256.f;        // 2^AT_SLACK: largest sum of a half tile's weights before the row's reference moves

// Heads of more than 128 (of the 4-bit cache, whose raw tiles are small enough): one row tile, and rings as long as fits.
template <int DP>
struct PrShape {
    static constexpr int TILES = DP == 256 ? 1 : 2, ROWS = TILES * PR_ROWS;      // row tiles and rows of an item
    static constexpr int PANELS = DP / 64;                          // 128-byte columns of an operand row
    static constexpr int PANEL = 128 * 128;                         // bytes: 128 rows x 128
    static constexpr int OPERAND = PANELS * PANEL;
    static constexpr int RING = DP == 256 ? 2 : 3, RAW_RING = DP == 256 ? 1 : 4;      // converted and raw tiles: K, V, K, V, ...
    static constexpr int RAW = DP == 256 ? PR_KEYS * (DP / 2 + DP / 16) : PR_KEYS * DP;
    static constexpr int Q_AT = 0, T_AT = TILES * OPERAND, RAW_AT = T_AT + RING * OPERAND;
    static constexpr int SC_AT = RAW_AT + RAW_RING * RAW;           // scales of four tiles: 8 of K, 8 of V
    static constexpr int F_AT = SC_AT + 4 * 64;                      // score factor of a row, fp32
    static constexpr int BAR_AT = F_AT + 2 * PR_ROWS * 4;
    static constexpr int SMEM = BAR_AT + 304 + 1024;
    // tensor memory: S (and P) of the two tiles, then O of the two tiles
    static constexpr int S_COL = 0, O_COL = 256, TMEM = 512;
    static_assert(SMEM <= 227 * 1024 && O_COL + TILES * DP <= TMEM, "");
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

// The same for the 4-bit cache: one factor for all scores of a row, no value scales.
__device__ __forceinline__ float pr_max4(unsigned (&s)[PR_SUB / 32][32], float kf, int upto, int from) {
    float bm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < PR_SUB; c += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) bm[u] = fmaxf(bm[u], c + u > upto || c + u <= from ? -INFINITY : __uint_as_float(s[(c + u) >> 5][(c + u) & 31]));
    const float top = fmaxf(fmaxf(bm[0], bm[1]), fmaxf(bm[2], bm[3]));
    return top == -INFINITY ? -INFINITY : top * kf;                  // a factor of 0 makes no NaN of a half that is masked whole
}
template <bool EDGE>
__device__ __forceinline__ float pr_weights4(unsigned ts, unsigned (&s)[PR_SUB / 32][32], float kf, float ref, int upto, int from) {
    f32x2 sum[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
    const f32x2 off = pk2(-ref, -ref), kk = pk2(kf, kf);
#pragma unroll
    for (int c = 0; c < PR_SUB / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float e[2];
            upk2(fma2(pk2(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])), kk, off), e[0], e[1]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                e[u] = at_exp2(e[u]);
                if (EDGE && (32 * c + i + u > upto || 32 * c + i + u <= from)) e[u] = 0.f;
            }
            sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], pk2(e[0], e[1]));
            p[i / 2] = at_half2(e[0], e[1]);
        }
        pr_st16(ts + 16 * c, p);
    }
    float lo, hi;
    upk2(add2(sum[0], sum[1]), lo, hi);
    return lo + hi;
}

// The plan of the shares (items: a CTA's query rows), written by a kernel of its own.
struct PrWork {
    long long* prefix;           // [row tiles of all requests + 1] units of one head before the row tile
    int4* start;                 // [ctas] (row tile of all requests, head, unit) a share starts with; x < 0: no share
    long long* share;            // units of a share; units in all
    int ctas;
};
template <int ROWS>
__device__ __forceinline__ int pr_units(const AtArgs& a, int row_tile) {
    const int steps = at_item<ROWS, PR_KEYS>(a, row_tile).steps;
    return steps ? steps + PR_EXTRA : 0;
}
template <int ROWS>
__global__ void __launch_bounds__(1024)
kv8_prompt_plan_kernel(const AtArgs a, const PrWork w) {
    __shared__ long long warp_sum_at[32], total_at;
    const int n = a.row_tiles * a.g.requests, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    sb_let_next();
    long long before = 0;
    for (int base = 0; base < n; base += 1024) {
        const int i = base + threadIdx.x;
        const long long mine = i < n ? pr_units<ROWS>(a, i) : 0;
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

template <int TYPE, int DP, bool DIRECT>
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
    const int pitch = TYPE == AT_E2M1 ? kv4_code_pitch(D) : D, spitch = kv4_scale_pitch(D);        // bytes of a token's codes and scales
    AtWalk<S::ROWS, PR_KEYS, PR_EXTRA> wk;
    sb_after_previous();
    sb_let_next();                           // its blocks find room when these end, and wait for that
    if (DIRECT) {
        // an item of its own, the requests' last row tiles, which have the most keys, first
        const int i = blockIdx.x / a.g.heads, before = i / a.g.requests, row_tile = (i - before * a.g.requests + 1) * a.row_tiles - 1 - before;
        const AtItem it = at_item<S::ROWS, PR_KEYS>(a, row_tile);
        if (!it.steps || !wk.begin(a, it, row_tile, (int)blockIdx.x - i * a.g.heads, 0, 0, it.steps + PR_EXTRA)) return;
    } else {
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
        for (bool more = true; more && ok; more = !DIRECT && wk.next(a), ++tiles_all) {
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
                constexpr int CH = NI < 16 ? NI : 16;                  // of them side by side
#pragma unroll 1
                for (int i0 = 0; i0 < NI; i0 += CH) {
                    uint4 x[CH];
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const int rr = qt * PR_ROWS + (warp & 3) * 32 + (i0 + i) * RPI + sub, at = head0 + rr;
                        const int tok = a.by_group.quot(at);
                        x[i] = make_uint4(0, 0, 0, 0);
                        if (rr < it.nrow && 8 * c < D)
                            x[i] = *reinterpret_cast<const uint4*>(src + tok * a.q_token_stride + (at - tok * a.group) * a.q_head_stride);
                    }
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        uint32_t m = __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
#pragma unroll
                        for (int o = 1; o < LANES; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                        const float up = at_query_scale(max(m & 0xffffu, m >> 16)), by = at_signed(up, a.scale_log2);
                        const int rr = (warp & 3) * 32 + (i0 + i) * RPI + sub;
                        if (c == 0) factor[rr] = up;
                        *reinterpret_cast<uint4*>(q0 + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) =
                            make_uint4(at_half2(bf16lo(x[i].x) * by, bf16hi(x[i].x) * by), at_half2(bf16lo(x[i].y) * by, bf16hi(x[i].y) * by),
                                       at_half2(bf16lo(x[i].z) * by, bf16hi(x[i].z) * by), at_half2(bf16lo(x[i].w) * by, bf16hi(x[i].w) * by));
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(qready + qt));
            }
            const float fq = __fdiv_rn(fabsf(a.scale_log2), reinterpret_cast<const float*>(smem + S::F_AT)[r]) *
                             (TYPE == AT_E2M1 && a.k_head ? a.k_head[wk.head] : 1.f);
            // (a thread without a row has queries of zeros, and its results go nowhere)
            const int pos = it.rq.past + a.by_group.quot(row);
            // positions of the tile's first and last row decide which key tiles need a mask
            const int pos_lo = it.rq.past + a.by_group.quot(it.r0 + qt * PR_ROWS);
            const int pos_hi = it.rq.past + a.by_group.quot(it.r0 + min(it.nrow, (qt + 1) * PR_ROWS) - 1);
            const int k0 = it.lo + wk.step0 * PR_KEYS, k1 = min(it.hi, k0 + count * PR_KEYS);
            // the sums so far in another scale: the products of the half before this one have to be done
            auto rescale = [&](int n, float f) -> bool {
                if (!wait(odone + qt, 2 * tiles_mine + n - 1)) return false;
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
                return true;
            };
            float m = -INFINITY, l = 0.f, inv = 0.f;
            // After tiles without rows the scales' phase before this one need not have ended. It has once there are scores: a
            // tile's scales come before its keys are converted.
            if constexpr (TYPE != AT_E2M1) {
                if (skipped) ok = wait(sfull + 2 * qt, tiles_mine);
                skipped = false;
                ok = ok && wait(scfull + (base_all & 3), base_all >> 2);
            }
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
                const int upto = min(pos, k1 - 1) - key, from = a.window > 0 ? pos - a.window - key : -1;
                float sum = 0.f;
                if constexpr (TYPE == AT_E2M1) {
                    // as below, with one factor and no value scales
                    bool again = edge || __any_sync(0xffffffffu, m == -INFINITY);
                    t5_wait_ld();
                    if (!again) {
                        sum = pr_weights4<false>(ts + PR_SUB * u, s, fq, m, upto, from);
                        again = __any_sync(0xffffffffu, !(sum <= PR_LIMIT4));
                    }
                    if (again) {
                        const float mx = pr_max4(s, fq, upto, from);
                        const bool far = mx > m + AT4_FAR;
                        float f = 1.f;
                        if (far) {
                            const float ref = mx - AT4_UP;
                            f = at_exp2(m - ref);
                            m = ref;
                            l *= f;
                        }
                        if (__any_sync(0xffffffffu, far) && n > 0) {
                            ok = rescale(n, f);
                            if (!ok) break;
                        }
                        pr_wait_st();
                        sum = pr_weights4<true>(ts + PR_SUB * u, s, fq, m == -INFINITY ? 0.f : m, upto, from);
                    }
                } else {
                    const float4* scj = reinterpret_cast<const float4*>(sc + 16 * ((base_all + j) & 3) + PR_SUBBLOCKS * u);
                    const float4 k4 = scj[0], v4 = scj[PR_BLOCKS / 4];
                    const float kf[PR_SUBBLOCKS] = {k4.x * fq, k4.y * fq, k4.z * fq, k4.w * fq};
                    const float vmax = fmaxf(fmaxf(v4.x, v4.y), fmaxf(v4.z, v4.w));
                    // Where nothing is masked, the weights by the reference there is; their sum says whether it
                    // still does: no weight is above their sum. One above PR_LIMIT (or none: NaN), a mask, a
                    // first key or a value scale too large takes the other way, by the row's maximum.
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
                            ok = rescale(n, f);
                            if (!ok) break;
                        }
                        const float ref = m == -INFINITY ? 0.f : m;
                        const float vw[PR_SUBBLOCKS] = {v4.x * inv, v4.y * inv, v4.z * inv, v4.w * inv};
                        pr_wait_st();
                        sum = pr_weights<true>(ts + PR_SUB * u, s, kf, vw, ref, upto, from);
                    }
                }
                l += sum;
                pr_wait_st();
                t5_fence_before();
                __syncwarp();
                if (lane == 0) t5_bar_arrive(t5_smem(pfull + 2 * qt + u));
                if (TYPE != AT_E2M1 && u && j + 1 < count) ok = wait(scfull + ((base_all + j + 1) & 3), (base_all + j + 1) >> 2);
            }
            // ---- results ----
            if (ok) ok = wait(fin + qt, pieces);
            if (!ok) break;
            t5_fence_after();
            tiles_mine += count;
            ++pieces;
            const bool whole = DIRECT || count == it.steps;
            const int h0 = wk.head * a.group;
            const int64_t tok = it.rq.row0 + a.by_group.quot(row);
            const int h = h0 + a.by_group.rem(row);
            const float back = TYPE != AT_E2M1 ? at_power_inv(inv) : a.v_head ? a.v_head[wk.head] : 1.f, norm = whole ? at_norm(l) * back : back;
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
                            *reinterpret_cast<float4*>(a.part + ((slot * (D / 4) + (c + i) / 4) * S::ROWS + r) * 4) =
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
            } else if (real) a.part_ml[slot * S::ROWS + r] = make_float2(m, l);
            t5_fence_before();                                       // the sums are read before the next piece's products
        }
    } else if (warp < 12) {
        // ---- conversion: a thread takes one 16-byte piece of every PASS-th row of a tile ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_CONVERT));
        constexpr int PIECES = DP / 16, PASS = 128 / PIECES, NP = PR_KEYS / PASS;
        const int tid = threadIdx.x - 256, piece = tid % PIECES, krow = tid / PIECES;
        // n: converted tile of all, left: rows that were copied and belong to the request (the rest: zeros)
        [[maybe_unused]] auto convert4 = [&](int n, int left) {
            const unsigned src = t5_smem(smem + S::RAW_AT + n % S::RAW_RING * S::RAW) + (unsigned)(krow * pitch + 8 * piece);
            const unsigned ssrc = t5_smem(smem + S::RAW_AT + n % S::RAW_RING * S::RAW) + (unsigned)(PR_KEYS * DP / 2 + krow * spitch + piece);
            unsigned char* dst = smem + S::T_AT + n % S::RING * S::OPERAND + (piece >> 2) * S::PANEL;
            if (16 * piece >= D) left = 0;
            uint2 x[NP];
            uint32_t sb[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                x[i] = make_uint2(0, 0);
                sb[i] = 0;
                if (krow + PASS * i < left) {
                    x[i] = at_lds64(src + (unsigned)(PASS * i * pitch));
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sb[i]) : "r"(ssrc + (unsigned)(PASS * i * spitch)));
                }
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int kk = krow + PASS * i;
                // as below: the second panel's lanes the other way round
                const bool swap = (piece >> 2) != 0;
                const int c = 2 * (piece & 3);
                const uint32_t s2 = e4m3x2_to_f16x2(sb[i] | sb[i] << 8);
                uint32_t h[2][4];
                fp4_unpack8(swap ? x[i].y : x[i].x, h[0]);
                fp4_unpack8(swap ? x[i].x : x[i].y, h[1]);
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<uint4*>(dst + kk * 128 + (((swap != (u != 0) ? c + 1 : c) ^ (kk & 7)) << 4)) =
                        make_uint4(f16x2_mul(h[u][0], s2), f16x2_mul(h[u][1], s2), f16x2_mul(h[u][2], s2), f16x2_mul(h[u][3], s2));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                t5_bar_arrive(t5_smem(full + n % S::RING));
                t5_bar_arrive(t5_smem(raw_empty + n % S::RAW_RING));
            }
        };
        [[maybe_unused]] auto convert = [&](int n, int left) {
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
        const bool brings = TYPE != AT_E2M1 && warp == 8 && lane < 2 * PR_BLOCKS;
        bool ok = true;
        int n = 0;                                                   // converted tiles so far
        for (bool more = true; more && ok; more = !DIRECT && wk.next(a)) {
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
                if (TYPE != AT_E2M1 && warp == 8 && !(i & 1)) {
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
                if constexpr (TYPE == AT_E2M1) convert4(n, limit - (i >> 1) * PR_KEYS);
                else convert(n, limit - (i >> 1) * PR_KEYS);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PR_REGS_REST));
    }
    if (warp == 13) {
        // ---- copies: a tile is eight scale blocks, each contiguous in its page; lane i brings block i ----
        // (of the 4-bit cache codes and scales)
        const unsigned bytes = (unsigned)(SB_KV8_BLOCK * pitch), sbytes = TYPE == AT_E2M1 ? (unsigned)(SB_KV8_BLOCK * spitch) : 0u;
        bool ok = true;
        int issued = 0;
        for (bool more = true; more && ok; more = !DIRECT && wk.next(a)) {
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
                if (inside && !fine) sb_latch(a.st, SB_ERR_INVALID, a.g.family);
                const int64_t at = ((int64_t)entry * a.g.heads + wk.head) * a.g.page_tokens + slot;
                const unsigned blocks = (unsigned)__popc(__ballot_sync(0xffffffffu, fine));
                entry = entry_of(j + 1);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int rs = issued % S::RAW_RING;
                    ok = ok && wait(raw_empty + rs, issued / S::RAW_RING + 1);
                    if (!ok) break;
                    const unsigned bar = t5_smem(raw_full + rs);
                    if (TYPE == AT_E2M1 && inside && !fine) {
                        // no such page: zeros, where a scale that was left there could be no number
                        unsigned char* raw = smem + S::RAW_AT + rs * S::RAW;
                        for (unsigned i = 0; i < bytes; i += 16) *reinterpret_cast<uint4*>(raw + lane * bytes + i) = make_uint4(0, 0, 0, 0);
                        for (int i = 0; i < (int)sbytes; i += 16) *reinterpret_cast<uint4*>(raw + PR_KEYS * DP / 2 + lane * sbytes + i) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) t5_bar_expect(bar, blocks * (bytes + sbytes));
                    __syncwarp();
                    const unsigned dst = t5_smem(smem + S::RAW_AT + rs * S::RAW);
                    if (fine) t5_load_bulk(dst + (unsigned)lane * bytes, (u ? a.v : a.k) + at * pitch, bytes, bar);
                    if (TYPE == AT_E2M1 && fine)
                        t5_load_bulk(dst + (unsigned)(PR_KEYS * DP / 2) + (unsigned)lane * sbytes, (u ? a.v_scale4 : a.k_scale4) + at * spitch, sbytes, bar);
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
        for (bool more = true; more && ok; more = !DIRECT && wk.next(a)) {
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
    if (threadIdx.x == 0 && *abort_flag) sb_latch(a.st, SB_ERR_TIMEOUT, a.g.family);
}

// The pieces of an item that lies in several shares, in their order. Block (c, y): the item that the
// border before share c + 1 cuts, if no earlier border does; 32 of its rows, eight threads a row, a
// thread every eighth four columns. The chain of dependent reads (share, item, sums) is what a block
// takes, so all columns go through it together (a block per 32 columns took 20 us for 4
// requests of up to 1024 tokens). What the plan says is read before the products have ended.
template <int DP>
__global__ void __launch_bounds__(256)
kv8_prompt_sum_kernel(const AtArgs a, const PrWork w) {
    constexpr int NQ = DP / 32, ROWS = PrShape<DP>::ROWS;
    const int c = blockIdx.x + 1, D = a.g.dim;
    const int4 s = w.start[c];
    const long long share = w.share[0], from = c * share - s.z;      // the item's first unit of all
    // a border that lies before the first tile, or behind one that cuts the same item, has nothing to add
    bool mine = s.x >= 0 && s.z > PR_EXTRA;
    const int c0 = mine ? (int)((from + PR_EXTRA) / share) : 0;      // the share with its first tile
    mine = mine && c == c0 + 1;
    AtItem it{};
    if (mine) it = at_item<ROWS, PR_KEYS>(a, s.x);
    const int r = 32 * blockIdx.y + threadIdx.x / 8, quad0 = threadIdx.x % 8;
    sb_after_previous();
    if (!mine || r >= it.nrow) return;
    const int c1 = (int)((from + it.steps + PR_EXTRA - 1) / share);
    float m = -INFINITY, l = 0.f;
    float4 v[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x = c0; x <= c1; ++x) {
        // the first piece of that share, unless the item starts inside the share
        const int64_t slot = 2 * (int64_t)x + (from > x * share ? 1 : 0);
        const float2 ml = a.part_ml[slot * ROWS + r];
        float4 y[NQ];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (4 * (quad0 + 8 * q) < D)
                y[q] = *reinterpret_cast<const float4*>(a.part + ((slot * (D / 4) + quad0 + 8 * q) * ROWS + r) * 4);
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

// Whether every item has a CTA of its own, without plan, pieces and their sum. Always where items are short (128-key tiles); up to 32
// tiles where the CTAs end about together, the longest first: what equal shares would win is less than what plan and sum take, 10
// tiles. Heads of 128, query heads four times the cache's 8, us, in shares and so, 4 and 8 bits: 1 request of 200 tokens 20.1 and
// 15.4, 20.3 and 15.9; 8 of 400 67 and 55, 72 and 57; 1 of 1500 58 and 37, 61 and 39; 8 of 900 166 and 131, 182 and 137; 1 of 4000 183 and
// 154, 198 and 166; 1 of 512 behind 1500 (in shares by this rule) 45 and 44, 48 and 48; 4 of 1024 behind 4000 (the same) 325 and 318, 365 and 351.
// Heads of 64: 1 of 1500 47 and 34, 51 and 34; 8 of 900 128 and 118, 145 and 112; 1 of 4000 153 and 141, 172 and 144; 1 of 512 behind 1500
// 37 and 42, 39 and 43. Heads of 256, 4 bits: 1 of 200 25 and 19, 1 of 1500 137 and 95, 8 of 900 481 and 334.
template <int ROWS>
bool pr_direct(const sb_ctx* ctx, const AtArgs& a, int64_t items, int64_t max_new, int64_t max_len) {
    // Where most requests have fewer rows than the longest, most of these CTAs find nothing, a round of them in about 1 us: 63 requests of one
    // token and one of 900 (7000 such CTAs) 104 us and in shares 84, 15 and one of 500 (800) 38 and 47.
    const int64_t real = at_real(a, ROWS, items);
    if (items >= (1ll << 31) || items - real > 16 * (int64_t)ctx->sm_count) return false;
    int64_t keys = max_len;
    if (a.window > 0 && keys > (int64_t)a.window + ROWS / a.group + 1 + SB_KV8_BLOCK) keys = (int64_t)a.window + ROWS / a.group + 1 + SB_KV8_BLOCK;
    const int64_t steps = (keys + PR_KEYS - 1) / PR_KEYS;
    if (steps <= 8 || steps > 32) return steps <= 8;
    // the first row tiles of prompts have fewer keys than the last
    const int64_t less = a.window > 0 ? 0 : max_new / PR_KEYS, least = (steps > less ? steps - less : 0) + PR_EXTRA;
    const double rounds = (double)real / ctx->sm_count, even = rounds * (double)(steps + PR_EXTRA + least) / 2;
    const double last = (double)((real + ctx->sm_count - 1) / ctx->sm_count) - rounds;            // of a round that is empty
    return even + last * (double)least <= even + 10 && (double)(steps + PR_EXTRA) <= even + 10;
}

template <int TYPE, int DP>
sb_status prompt_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = PrShape<DP>;
    const int64_t row_tiles = (max_new * a.group + S::ROWS - 1) / S::ROWS, n = row_tiles * a.g.requests;
    if (n >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "%s attention: too many query rows", TYPE == AT_E2M1 ? "kv4" : "kv8");
    int64_t keys = max_len;
    if (a.window > 0 && keys > a.window + max_new + PR_KEYS) keys = a.window + max_new + PR_KEYS;
    // one share per SM, fewer if there cannot be so many shares
    const int64_t most = (n * a.g.heads * ((keys + PR_KEYS - 1) / PR_KEYS + 1 + PR_EXTRA) + PR_LEAST - 1) / PR_LEAST;
    PrWork w{};
    w.ctas = (int)(most < ctx->sm_count ? most : ctx->sm_count);
    a.row_tiles = (int)row_tiles;
    a.by_row_tiles = KvDiv(a.row_tiles);
    a.direct = pr_direct<S::ROWS>(ctx, a, n * a.g.heads, max_new, max_len);
    auto* kernel = a.direct ? kv8_prompt_kernel<TYPE, DP, true> : kv8_prompt_kernel<TYPE, DP, false>;
    if (a.direct) return sb_launch(ctx, kernel, dim3((unsigned)(n * a.g.heads)), PR_THREADS, S::SMEM, 1, true, a, w);
    const size_t rows = (size_t)w.ctas * 2 * S::ROWS;
    void* arena;
    const sb_status s = sb_scratch(ctx, Carver::need({((size_t)n + 1) * 8, (size_t)w.ctas * 16, 16, rows * a.g.dim * 4, rows * 8}), &arena);
    if (s != SB_OK) return s;
    Carver cv(arena);
    w.prefix = cv.take<long long>((size_t)n + 1);
    w.start = cv.take<int4>(w.ctas);
    w.share = cv.take<long long>(2);
    a.part = cv.take<float>(rows * a.g.dim);
    a.part_ml = cv.take<float2>(rows);
    kv8_prompt_plan_kernel<S::ROWS><<<1, 1024, 0, ctx->stream>>>(a, w);
    SB_LAUNCHED(ctx);
    // The other two are sent off while the kernel before them still runs and wait on the device for its
    // end, which hides their launches.
    const sb_status t = sb_launch(ctx, kernel, dim3((unsigned)w.ctas), PR_THREADS, S::SMEM, 1, true, a, w);
    if (t != SB_OK || w.ctas <= 1) return t;
    return sb_launch(ctx, kv8_prompt_sum_kernel<DP>, dim3((unsigned)(w.ctas - 1), S::ROWS / 32), 256, 0, 1, true, a, w);
}

}  // namespace

sb_status kv8_prompt(sb_ctx* ctx, AtArgs a, int type, int64_t max_new, int64_t max_len) {
    if (type == AT_E2M1)
        return a.g.dim <= 64 ? prompt_launch<AT_E2M1, 64>(ctx, a, max_new, max_len)
             : a.g.dim <= 128 ? prompt_launch<AT_E2M1, 128>(ctx, a, max_new, max_len) : prompt_launch<AT_E2M1, 256>(ctx, a, max_new, max_len);
    if (type == SB_KV_INT8)
        return a.g.dim <= 64 ? prompt_launch<SB_KV_INT8, 64>(ctx, a, max_new, max_len) : prompt_launch<SB_KV_INT8, 128>(ctx, a, max_new, max_len);
    return a.g.dim <= 64 ? prompt_launch<SB_KV_E4M3, 64>(ctx, a, max_new, max_len) : prompt_launch<SB_KV_E4M3, 128>(ctx, a, max_new, max_len);
}
