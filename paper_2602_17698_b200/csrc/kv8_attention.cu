// Attention of a few query rows over the 8-bit cache: decode steps and drafted tokens.
//
// A cache head is read once for all its query rows (new tokens x query heads that share it): NR
// tiles of 8 rows.  Per 16 keys the two products run on mma.sync m16n8k16 (fp16 operands, fp32
// sums) with the KEYS on the 16-row side, so that 8 query rows fill an instruction:
//     S^T[key][row] = K Q^T,     O^T[d][row] += V^T P^T,
// and a tile of 16 keys is one scale block: its key scale multiplies 16 x 8 scores, its value
// scale 16 x 8 weights.  The arithmetic needs a third of the tensor pipe's time at the rate the
// cache can be read; what bounds the kernel is that read, so everything is arranged to keep
// copies in flight: every warp has a ring of its own in shared memory, filled by 16-byte cp.async
// (zero-filled past the request's end, so nothing stale reaches a product), and no warp waits for
// another before the end of its chunk.
//
// Codes go from shared memory into operand registers without a transposition:
//   K: the contraction over d may visit d in any order, so lane (g, t) of the A operand takes 16
//      consecutive d of rows g and g + 8 with one 16-byte load: four steps of the contraction.
//   V: lane (g, t) takes 16 consecutive d of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9; byte c of two
//      keys, side by side, is a pair of the A operand of V^T for d = 16 g + c.
// 16-byte pieces of a row are XOR-ed with the row number, which makes both loads conflict-free.
// e4m3 pairs become fp16 by one conversion; an int8 byte with the sign bit flipped is put under
// the exponent of 1024 (1152 + code) and 1152 is subtracted: exact.
//
// Precision: a query row is scaled by a power of two to at most 2^14 and held in fp16 (exact for
// every element above 2^-28 of the row's largest), scores and sums are fp32, the weight of a key
// times its value scale, relative to a power of two of its row, is rounded to fp16 (2^-11): three
// bits finer than the bf16 result. That rounding is nearly all by which results differ from a form in
// fp32 (0.0008 of their norm for 64 requests in 8192; both are 0.0017 from 64 bits, bf16's rounding).
//
// The work of all requests is cut into equal shares (see kv8_attention.cuh), which every CTA finds by
// itself from the requests' lengths. Of an item that several shares hold, each leaves unnormalised sums,
// and the last of them to finish (a counter) adds them in their order: the result does not depend on
// which one that is.
//
// Measured (heads of 128, four query heads per cache head, 8 cache heads): 64 requests in 8192 88 us, 5.7 TB/s, 0.88
// of a plain copy's rate; one in 100000 47 us, of which 35 stream at 5.9 TB/s and the rest is the start and the
// sum of the pieces; 16 x 5 tokens in a window of 4096 (20 rows) 58 us: 251 registers leave two warps a scheduler,
// and their latencies bound it.
#include "kv8_attention.cuh"

namespace {

// More query rows than this per cache head go to the tcgen05 kernel, which takes 256 at the price of one. Heads of 128,
// four query rows per token: 4 requests in 200 tokens 19 us there, 26, 39 and 47 here with 12, 24 and 32 rows; one in 8192
// 37 and 51 with 24 rows, 39 and 68 with 32; but 16 in 2000 58 and 44 with 24 rows, 63 and 62 with 32. So rows alone do
// not decide it: few requests would gain from the other kernel below 24 rows already, many lose until 32; the limit
// is near where many requests change sides. Heads of more than 128 have no kernel there: all their rows run here.
constexpr int AT_PROMPT_FROM = 24;
constexpr int AT_WARPS = 4;
constexpr int AT_STEP = 32;             // keys a warp takes at a time: two scale blocks
constexpr int AT_EXTRA = 12;            // what an item costs besides its steps, in steps
constexpr int AT_BATCH = 16;            // steps whose page numbers and scales a warp holds, two lanes a step

__device__ __forceinline__ unsigned at_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void at_copy16(unsigned dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void at_copy16(unsigned dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void at_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void at_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void at_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t at_transpose(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <int DP, int NR>
struct AtShape {
    static constexpr int STAGES = DP == 64 ? 4 : NR == 1 ? 2 : 3;
    static constexpr int CTAS = DP == 256 ? 1 : NR == 1 ? 3 : 2;     // resident per SM: registers and the rings decide
    static constexpr int SIDE = AT_STEP * DP;                      // bytes of a step's keys
    static constexpr int RING = AT_WARPS * STAGES * 2 * SIDE;
    static constexpr int ROWS = 8 * NR;
    static constexpr int QPITCH = 2 * DP + 16;                     // bytes of a query row
    static constexpr int Q_AT = RING;
    static constexpr int F_AT = Q_AT + ROWS * QPITCH;              // score factor of a row, fp32
    static constexpr int FLAG_AT = F_AT + ROWS * 4;
    static constexpr int SMEM = FLAG_AT + 64;
    static constexpr int OPITCH = DP + 4;                          // floats of a row of a warp's sums
    static_assert(AT_WARPS * ROWS * (OPITCH + 2) * 4 <= RING, "the warps' sums fit where the ring was");
    static_assert(CTAS * 160 * ROWS * 4 + AT_WARPS * 32 * 16 <= RING && QPITCH >= 8, "so do the weights of an item's pieces");
    static constexpr bool QREGS = NR * DP <= 256;                  // query operands stay in registers
};

template <int TYPE, int DP, int NR>
__global__ void __launch_bounds__(AT_WARPS * 32, AtShape<DP, NR>::CTAS)
kv8_rows_kernel(const AtArgs a) {
    using S = AtShape<DP, NR>;
    constexpr int KS = DP / 16;                    // contraction steps over d
    constexpr int MT = DP / 16;                    // 16-row tiles of O^T
    constexpr int PIECES = DP / 16;                // 16-byte pieces of a row
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int D = a.g.dim;
    // ---- this CTA's share ----
    AtWalk<S::ROWS, AT_STEP, AT_EXTRA> wk;
    long long share;
    {
        // units of one head before each row tile of all requests, 128 at a time
        long long* sums = reinterpret_cast<long long*>(smem);       // [AT_WARPS] and, behind them, where the share starts
        const int n = a.row_tiles * a.g.requests;
        auto units = [&](int i) -> long long {
            if (i >= n) return 0;
            const int steps = at_item<S::ROWS, AT_STEP>(a, i).steps;
            return steps ? steps + AT_EXTRA : 0;
        };
        long long mine = units(threadIdx.x), x = mine;
        for (int i = threadIdx.x + AT_WARPS * 32; i < n; i += AT_WARPS * 32) x += units(i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane == 0) sums[warp] = x;
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int w = 0; w < AT_WARPS; ++w) total += sums[w];
        total *= a.g.heads;
        share = at_div(total + gridDim.x - 1, gridDim.x);
        if (share < a.least) share = a.least;
        const long long at = blockIdx.x * share;
        if (at >= total) return;
        long long before = 0;
        for (int base = 0; base < n; base += AT_WARPS * 32) {
            if (base > 0) mine = units(base + threadIdx.x);
            x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            __syncthreads();
            if (lane == 31) sums[warp] = x;
            __syncthreads();
            long long all = 0, below = before;
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) {
                if (w < warp) below += sums[w];
                all += sums[w];
            }
            const long long lo = (below + x - mine) * a.g.heads;     // the row tile's first unit of all
            if (at >= lo && at < lo + mine * a.g.heads) {
                int* found = reinterpret_cast<int*>(sums + AT_WARPS);
                found[0] = base + threadIdx.x;
                found[1] = (int)at_div(at - lo, mine);
                found[2] = (int)(at - lo - found[1] * mine);
            }
            before += all;
            if (at < before * a.g.heads) break;
        }
        __syncthreads();
        const int* found = reinterpret_cast<const int*>(sums + AT_WARPS);
        const int f0 = found[0], f1 = found[1], f2 = found[2];
        __syncthreads();
        if (!wk.begin(a, f0, f1, f2, at, min(share, total - at))) return;
    }
    for (bool more = true; more; more = wk.next(a)) {
        const int head = wk.head, b = wk.it.b, r0 = wk.it.r0, nrow = wk.it.nrow;
        const Kv8Request rq = wk.it.rq;
        const int i0 = a.by_group.quot(r0), i1 = a.by_group.quot(r0 + nrow - 1);
        const int k0 = wk.it.lo + wk.step0 * AT_STEP, k1 = min(wk.it.hi, k0 + wk.count * AT_STEP);
        const int mine = (wk.count - warp + AT_WARPS - 1) / AT_WARPS;   // steps warp, warp + 4, ...

        // the queries are on their way before the chain of table, scales and codes begins
        constexpr int QR = S::ROWS / AT_WARPS;
        uint32_t qw[QR][DP / 64];
#pragma unroll
        for (int i = 0; i < QR; ++i) {
            const int r = warp + AT_WARPS * i, row = r0 + r;
            const __nv_bfloat16* src = a.q + (int64_t)(rq.row0 + a.by_group.quot(row)) * a.q_token_stride +
                                       (int64_t)(head * a.group + a.by_group.rem(row)) * a.q_head_stride;
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) {
                const int d = 64 * c + 2 * lane;
                qw[i][c] = r < nrow && d < D ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
            }
        }

        // ---- where this warp's blocks lie and their scales, AT_BATCH steps at a time: lane 2 s + e holds block e
        // of step s; the table's entries are fetched two batches ahead, scales one ----
        auto block_key = [&](int batch) { return k0 + (warp + AT_WARPS * (AT_BATCH * batch + (lane >> 1))) * AT_STEP + SB_KV8_BLOCK * (lane & 1); };
        auto load_entry = [&](int batch) -> int {
            const int key = block_key(batch);
            return key < k1 ? a.g.table[(int64_t)b * a.g.table_stride + a.g.page.quot(key)] : 0;
        };
        // the block's first code (-1: no such block) and, fetched, its two scales
        auto place = [&](int batch, int entry, uint32_t& s2) -> int64_t {
            const int key = block_key(batch);
            s2 = 0;
            if (key >= k1) return -1;
            if (entry < 0 || entry >= a.g.pages) {
                sb_latch(a.st, SB_ERR_INVALID, SBK_KV8);
                return -1;
            }
            const int64_t ph = (int64_t)entry * a.g.heads + head;
            const int slot = a.g.page.rem(key);
            const int64_t at = ph * (a.g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK;
            s2 = (uint32_t)a.k_scale[at] | (uint32_t)a.v_scale[at] << 16;
            return (ph * a.g.page_tokens + slot) * D;
        };
        int entry_next = load_entry(1);
        uint32_t sc_cur, sc_next = 0;
        int64_t at_even = place(0, load_entry(0), sc_cur), at_odd = -1;     // of even and odd batches

        const unsigned ring = at_smem(smem) + (unsigned)(warp * S::STAGES * 2 * S::SIDE);
        // copies of step j of this warp into its ring
        constexpr int TOKS = 32 / PIECES;                               // tokens a warp copies with one instruction
        const int cp_piece = lane % PIECES, cp_tok = lane / PIECES;
        const int cp_off = cp_tok * D + cp_piece * 16;
        auto ring_at = [](int row, int piece) {
            return DP == 64 ? (unsigned)(row * 64 + ((piece ^ ((row >> 1) & 3)) << 4)) : (unsigned)(row * DP + ((piece ^ (row & 7)) << 4));
        };
        auto issue = [&](int j) {
            if (j < mine) {
                const int key = k0 + (warp + AT_WARPS * j) * AT_STEP;
                const unsigned dst = ring + (unsigned)((j % S::STAGES) * 2 * S::SIDE);
                const int64_t held = (j / AT_BATCH) & 1 ? at_odd : at_even;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int64_t base = __shfl_sync(0xffffffffu, held, 2 * (j & (AT_BATCH - 1)) + e);
                    const uint8_t *kp = a.k + base + cp_off, *vp = a.v + base + cp_off;
                    if (D == DP && base >= 0 && key + SB_KV8_BLOCK * (e + 1) <= rq.len) {
#pragma unroll
                        for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) {
                            const unsigned to = ring_at(SB_KV8_BLOCK * e + cp_tok + TOKS * i, cp_piece);
                            at_copy16(dst + to, kp + TOKS * i * DP);
                            at_copy16(dst + S::SIDE + to, vp + TOKS * i * DP);
                        }
                    } else {
                        // the last block, a block that is not there, or rows shorter than the operand's: zeros fill up
#pragma unroll
                        for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) {
                            const int tok = cp_tok + TOKS * i;
                            const bool take = base >= 0 && key + SB_KV8_BLOCK * e + tok < rq.len && cp_piece * 16 < D;
                            const unsigned to = ring_at(SB_KV8_BLOCK * e + tok, cp_piece);
                            at_copy16(dst + to, take ? kp + TOKS * i * D : a.k, take);
                            at_copy16(dst + S::SIDE + to, take ? vp + TOKS * i * D : a.v, take);
                        }
                    }
                }
            }
            at_commit();
        };
#pragma unroll
        for (int j = 0; j < S::STAGES - 1; ++j) issue(j);

        // ---- queries: fp16 rows, each scaled by a power of two ----
#pragma unroll
        for (int i = 0; i < QR; ++i) {
            const int r = warp + AT_WARPS * i;
            unsigned char* qrow = smem + S::Q_AT + r * S::QPITCH;
            uint32_t amax = 0;
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) amax = max(amax, max(qw[i][c] & 0x7fffu, (qw[i][c] >> 16) & 0x7fffu));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const float up = at_query_scale(amax), by = at_signed(up, a.scale_log2);
#pragma unroll
            for (int c = 0; c < DP / 64; ++c)
                *reinterpret_cast<uint32_t*>(qrow + 128 * c + 4 * lane) = at_half2(bf16lo(qw[i][c]) * by, bf16hi(qw[i][c]) * by);
            if (lane == 0) reinterpret_cast<float*>(smem + S::F_AT)[r] = __fdiv_rn(fabsf(a.scale_log2), up);
        }
        __syncthreads();
        float fq[NR][2];
        int pos[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * nr + 2 * t + e;
                fq[nr][e] = reinterpret_cast<const float*>(smem + S::F_AT)[r];
                pos[nr][e] = rq.past + a.by_group.quot(r0 + r);          // rows past the last: queries of zeros, dropped at the end
            }
        // B operand of step 4 c + j: d = 64 c + 16 t + 4 j + {0, 1} and + {2, 3} of row g
        const unsigned qlane = at_smem(smem) + S::Q_AT + (unsigned)(g * S::QPITCH + 32 * t);
        uint2 qf[S::QREGS ? KS : 1][NR];
        if (S::QREGS) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) qf[s][nr] = at_lds64(qlane + (unsigned)(8 * nr * S::QPITCH + 128 * (s >> 2) + 8 * (s & 3)));
        }

        float o[MT][NR][4], m[NR][2], l[NR][2], inv[NR][2];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) o[i][nr][0] = o[i][nr][1] = o[i][nr][2] = o[i][nr][3] = 0.f;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[nr][e] = -INFINITY; l[nr][e] = inv[nr][e] = 0.f; }

        for (int j = 0; j < mine; ++j) {
            if ((j & (AT_BATCH - 1)) == 0) {
                const int batch = j / AT_BATCH;
                if (batch > 0) sc_cur = sc_next;
                if (AT_BATCH * (batch + 1) < mine) {
                    const int64_t at = place(batch + 1, entry_next, sc_next);
                    if (batch & 1) at_even = at;                         // the slot of the batch before this one
                    else at_odd = at;
                    entry_next = load_entry(batch + 2);
                }
            }
            at_wait<S::STAGES - 2>();
            __syncwarp();
            issue(j + S::STAGES - 1);
            const int key = k0 + (warp + AT_WARPS * j) * AT_STEP;
            const unsigned kst = ring + (unsigned)((j % S::STAGES) * 2 * S::SIDE), vst = kst + S::SIDE;
            float ksc[2], vsc[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t s2 = __shfl_sync(0xffffffffu, sc_cur, 2 * (j & (AT_BATCH - 1)) + e);
                ksc[e] = __uint_as_float(s2 << 16);
                vsc[e] = __uint_as_float(s2 & 0xffff0000u);
            }
            // scores, in units of log2
            float s[2][NR][4];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) s[e][nr][0] = s[e][nr][1] = s[e][nr][2] = s[e][nr][3] = 0.f;
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) {
                // both blocks side by side: twice the independent products, one fetch of the queries for both
                uint32_t wl[2][4], wh[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = SB_KV8_BLOCK * e + g;           // rows g and g + 8 have the same swizzle
                    const unsigned off = DP == 64 ? (unsigned)(row * 64 + ((t ^ ((row >> 1) & 3)) << 4))
                                                  : (unsigned)(row * DP + 128 * (c >> 1) + (((4 * (c & 1) + t) ^ (row & 7)) << 4));
                    const uint4 lo4 = at_lds128(kst + off), hi4 = at_lds128(kst + off + 8 * DP);
                    wl[e][0] = at_flip<TYPE>(lo4.x); wl[e][1] = at_flip<TYPE>(lo4.y); wl[e][2] = at_flip<TYPE>(lo4.z); wl[e][3] = at_flip<TYPE>(lo4.w);
                    wh[e][0] = at_flip<TYPE>(hi4.x); wh[e][1] = at_flip<TYPE>(hi4.y); wh[e][2] = at_flip<TYPE>(hi4.z); wh[e][3] = at_flip<TYPE>(hi4.w);
                }
                uint4 q4[2][NR];
                if constexpr (!S::QREGS) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) q4[h][nr] = at_lds128(qlane + (unsigned)(8 * nr * S::QPITCH + 128 * c + 16 * h));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t x = wl[e][i], y = wh[e][i];
                        const uint32_t a0 = at_pair<TYPE, 0>(x), a1 = at_pair<TYPE, 0>(y), a2 = at_pair<TYPE, 1>(x), a3 = at_pair<TYPE, 1>(y);
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) {
                            uint2 qb;
                            if constexpr (S::QREGS) qb = qf[4 * c + i][nr];
                            else qb = i & 1 ? make_uint2(q4[i >> 1][nr].z, q4[i >> 1][nr].w) : make_uint2(q4[i >> 1][nr].x, q4[i >> 1][nr].y);
                            at_mma(s[e][nr], a0, a1, a2, a3, qb.x, qb.y);
                        }
                    }
                }
            }
            const float vmax = fmaxf(vsc[0], vsc[1]);
            const bool edge = key + AT_STEP > rq.past + i0 + 1 || key + AT_STEP > k1 || (a.window > 0 && key <= rq.past + i1 - a.window);
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = s[e][nr][i] * (ksc[e] * fq[nr][i & 1]);
                        if (edge) {
                            const int kk = key + SB_KV8_BLOCK * e + g + 8 * (i >> 1), p = pos[nr][i & 1];
                            if (kk > p || kk >= k1 || (a.window > 0 && kk <= p - a.window)) x = -INFINITY;
                        }
                        s[e][nr][i] = x;
                        mx[i & 1] = fmaxf(mx[i & 1], x);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], w));
                }
                // the reference only moves when it is off by more than 2^8: a weight stays below 2^8
                bool off[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    off[e] = mx[e] > m[nr][e] + AT_SLACK || (m[nr][e] == -INFINITY && mx[e] > m[nr][e]) || vmax * inv[nr][e] > AT_TOP;
                if (__any_sync(0xffffffffu, off[0] || off[1])) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float ref = fmaxf(m[nr][e], mx[e]);
                        // the row's largest weight times value scale, block by block
                        float most = 0.f;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float top = fmaxf(s[k][nr][e], s[k][nr][2 + e]);
#pragma unroll
                            for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                            most = fmaxf(most, at_exp2(top - ref) * vsc[k]);
                        }
                        f[e] = 1.f;
                        if (off[e]) {
                            const float down = m[nr][e] == -INFINITY ? 0.f : at_exp2(m[nr][e] - ref), held = at_power_inv(inv[nr][e]) * down;
                            inv[nr][e] = at_value_inv(most, held, vmax);
                            m[nr][e] = ref;
                            l[nr][e] *= down;
                            f[e] = held * inv[nr][e];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[i][nr][0] *= f[0]; o[i][nr][1] *= f[1]; o[i][nr][2] *= f[0]; o[i][nr][3] *= f[1];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint32_t pb[NR][2];
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) {
                    const float vw[2] = {vsc[e] * inv[nr][0], vsc[e] * inv[nr][1]};
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float mm = m[nr][i & 1];
                        p[i] = at_exp2(s[e][nr][i] - (mm == -INFINITY ? 0.f : mm));
                        l[nr][i & 1] += p[i];
                    }
                    pb[nr][0] = at_transpose(at_half2(p[0] * vw[0], p[1] * vw[1]));
                    pb[nr][1] = at_transpose(at_half2(p[2] * vw[0], p[3] * vw[1]));
                }
                constexpr int VP = DP / 128 > 0 ? DP / 128 : 1;          // panels of 128 d
                constexpr int VW = DP == 64 ? 2 : 4;                     // words a lane takes of a row and panel
#pragma unroll
                for (int pn = 0; pn < VP; ++pn) {
                    uint32_t w[4][VW];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = SB_KV8_BLOCK * e + 2 * t + (k & 1) + 8 * (k >> 1);
                        if constexpr (DP == 64) {
                            const uint2 x = at_lds64(vst + (unsigned)(row * 64 + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + 8 * (g & 1)));
                            w[k][0] = at_flip<TYPE>(x.x); w[k][1] = at_flip<TYPE>(x.y);
                        } else {
                            const uint4 x = at_lds128(vst + (unsigned)(row * DP + 128 * pn + ((g ^ (row & 7)) << 4)));
                            w[k][0] = at_flip<TYPE>(x.x); w[k][1] = at_flip<TYPE>(x.y);
                            w[k][2] = at_flip<TYPE>(x.z); w[k][3] = at_flip<TYPE>(x.w);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < VW; ++c) {
                        // bytes 0, 1 and 2, 3 of the two key pairs, interleaved
                        const uint32_t l01 = __byte_perm(w[0][c], w[1][c], 0x5140), l23 = __byte_perm(w[0][c], w[1][c], 0x7362);
                        const uint32_t h01 = __byte_perm(w[2][c], w[3][c], 0x5140), h23 = __byte_perm(w[2][c], w[3][c], 0x7362);
                        const uint32_t a0 = at_pair<TYPE, 0>(l01), a1 = at_pair<TYPE, 1>(l01), a2 = at_pair<TYPE, 0>(h01), a3 = at_pair<TYPE, 1>(h01);
                        const uint32_t c0 = at_pair<TYPE, 0>(l23), c1 = at_pair<TYPE, 1>(l23), c2 = at_pair<TYPE, 0>(h23), c3 = at_pair<TYPE, 1>(h23);
                        const int i = 2 * (VW * pn + c);
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) {
                            at_mma(o[i][nr], a0, a1, a2, a3, pb[nr][0], pb[nr][1]);
                            at_mma(o[i + 1][nr], c0, c1, c2, c3, pb[nr][0], pb[nr][1]);
                        }
                    }
                }
            }
        }
        at_wait<0>();
        __syncthreads();

        // ---- the warps' sums side by side where the ring was ----
        float* osm = reinterpret_cast<float*>(smem);                     // [warp][row][OPITCH]
        float2* mlsm = reinterpret_cast<float2*>(smem + (size_t)AT_WARPS * S::ROWS * S::OPITCH * 4);      // [warp][row]
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nr][e];
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                const int r = 8 * nr + 2 * t + e;
                if (g == 0) mlsm[warp * S::ROWS + r] = make_float2(m[nr][e], sum);
                float* row = osm + (warp * S::ROWS + r) * S::OPITCH;
                const float back = at_power_inv(inv[nr][e]);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    // o[i][.][e] and [2 + e]: two neighbouring d of row r
                    constexpr int LW = DP == 64 ? 8 : 16;                // d a lane holds per panel
                    const int d = LW * g + 128 * (i / (LW / 2)) + 2 * (i % (LW / 2));
                    *reinterpret_cast<float2*>(row + d) = make_float2(o[i][nr][e] * back, o[i][nr][2 + e] * back);
                }
            }
        __syncthreads();
        const bool whole = wk.count == wk.it.steps;
        const int quads = D / 4;
        auto store = [&](int r, int d, float4 v, float mm, float sum) {
            const int row = r0 + r;
            const int64_t tok = rq.row0 + a.by_group.quot(row);
            const int h = head * a.group + a.by_group.rem(row);
            const float f = at_norm(sum);
            const uint2 w = make_uint2(u32(__floats2bfloat162_rn(v.x * f, v.y * f)), u32(__floats2bfloat162_rn(v.z * f, v.w * f)));
            *reinterpret_cast<uint2*>(a.o + tok * a.o_token_stride + h * a.o_head_stride + d) = w;
            if (d == 0 && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(mm, sum);
        };
        for (int idx = threadIdx.x; idx < nrow * quads; idx += AT_WARPS * 32) {
            const int r = idx / quads, d = 4 * (idx - r * quads);
            float2 ml[AT_WARPS];
            float mm = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) {
                ml[w] = mlsm[w * S::ROWS + r];
                mm = fmaxf(mm, ml[w].x);
            }
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) {
                const float f = ml[w].x == -INFINITY ? 0.f : at_exp2(ml[w].x - mm);
                const float4 x = *reinterpret_cast<const float4*>(osm + (w * S::ROWS + r) * S::OPITCH + d);
                sum = fmaf(ml[w].y, f, sum);
                v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
            }
            if (whole) store(r, d, v, mm, sum);
            else {
                const int64_t at = (2 * (int64_t)blockIdx.x + (wk.first ? 0 : 1)) * S::ROWS + r;
                *reinterpret_cast<float4*>(a.part + at * D + d) = v;
                if (d == 0) a.part_ml[at] = make_float2(mm, sum);
            }
        }
        if (!whole) {
            // ---- the last of the item's pieces to finish adds them all, in order ----
            const long long from = wk.from;
            const int c0 = (int)at_div(from + AT_EXTRA, share), c1 = (int)at_div(from + wk.units() - 1, share), pieces = c1 - c0 + 1;
            // a piece is the first of its share unless the item starts inside the share
            auto slot = [&](int x) { return (2 * (int64_t)(c0 + x) + (from > (c0 + x) * share ? 1 : 0)) * S::ROWS; };
            volatile int* last = reinterpret_cast<volatile int*>(smem + S::FLAG_AT);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                unsigned* done = a.done + ((int64_t)wk.row_tile * a.g.heads + head);
                *last = atomicAdd(done, 1u) == (unsigned)(pieces - 1);
                if (*last) *done = 0;                                    // for the next call
            }
            __syncthreads();
            if (*last) {
                __threadfence();
                // weights of the pieces of every row in shared memory, a row per warp
                float* weight = reinterpret_cast<float*>(smem);          // [pieces][ROWS]
                float2* total = reinterpret_cast<float2*>(smem + S::F_AT - S::ROWS * 8);         // (reference, sum) of a row
                for (int r = warp; r < nrow; r += AT_WARPS) {
                    constexpr int HELD = 4;                              // of a lane's pieces in registers: 128 in all
                    float2 ml[HELD];
                    float mm = -INFINITY, sum = 0.f;
#pragma unroll
                    for (int i = 0; i < HELD; ++i) {
                        const int x = lane + 32 * i;
                        ml[i] = x < pieces ? __ldcg(a.part_ml + slot(x) + r) : make_float2(-INFINITY, 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < HELD; ++i) mm = fmaxf(mm, ml[i].x);
                    for (int x = lane + 32 * HELD; x < pieces; x += 32) mm = fmaxf(mm, __ldcg(a.part_ml + slot(x) + r).x);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, o));
                    auto put = [&](int x, float2 p) {
                        const float f = p.x == -INFINITY ? 0.f : at_exp2(p.x - mm);
                        weight[x * S::ROWS + r] = f;
                        sum = fmaf(p.y, f, sum);
                    };
#pragma unroll
                    for (int i = 0; i < HELD; ++i)
                        if (lane + 32 * i < pieces) put(lane + 32 * i, ml[i]);
                    for (int x = lane + 32 * HELD; x < pieces; x += 32) put(x, __ldcg(a.part_ml + slot(x) + r));
                    sum = warp_sum(sum);
                    if (lane == 0) total[r] = make_float2(mm, sum);
                }
                __syncthreads();
                constexpr int PER = S::ROWS * DP / 4 / (AT_WARPS * 32);  // outputs of a thread, four columns each, at most
                const int outs = nrow * quads;
                if (outs <= AT_WARPS * 32) {
                    // few outputs: one a thread, or several threads for one, each a part of the pieces
                    const int parts = AT_WARPS * 32 / outs, part = (int)threadIdx.x / outs, idx = (int)threadIdx.x - part * outs;
                    const int r = idx / quads, d = 4 * (idx - r * quads);
                    float4* shared_sum = reinterpret_cast<float4*>(smem + (S::RING - AT_WARPS * 32 * 16));
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (part < parts) {
                        const int x1 = pieces * (part + 1) / parts;
#pragma unroll 8
                        for (int x = pieces * part / parts; x < x1; ++x) {
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part + (slot(x) + r) * D + d));
                            const float f = weight[x * S::ROWS + r];
                            v.x = fmaf(y.x, f, v.x); v.y = fmaf(y.y, f, v.y); v.z = fmaf(y.z, f, v.z); v.w = fmaf(y.w, f, v.w);
                        }
                    }
                    shared_sum[threadIdx.x] = v;
                    __syncthreads();
                    if ((int)threadIdx.x < outs) {
                        for (int p = 1; p < parts; ++p) {
                            const float4 y = shared_sum[threadIdx.x + p * outs];
                            v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
                        }
                        store(r, d, v, total[r].x, total[r].y);
                    }
                } else {
                    // a thread's outputs side by side, so that their loads overlap
                    float4 v[PER];
#pragma unroll
                    for (int i = 0; i < PER; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll (PER <= 2 ? 8 : 2)
                    for (int x = 0; x < pieces; ++x) {
                        const float* from_part = a.part + slot(x) * D;
#pragma unroll
                        for (int i = 0; i < PER; ++i) {
                            const int idx = (int)threadIdx.x + AT_WARPS * 32 * i;
                            if (idx >= outs) continue;
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(from_part) + idx);
                            const float f = weight[x * S::ROWS + idx / quads];
                            v[i].x = fmaf(y.x, f, v[i].x); v[i].y = fmaf(y.y, f, v[i].y); v[i].z = fmaf(y.z, f, v[i].z); v[i].w = fmaf(y.w, f, v[i].w);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const int idx = (int)threadIdx.x + AT_WARPS * 32 * i, r = idx / quads;
                        if (idx < outs) store(r, 4 * (idx - r * quads), v[i], total[r].x, total[r].y);
                    }
                }
            }
        }
        __syncthreads();                                                 // the next piece's copies go where the sums were
    }
}

template <int TYPE, int DP, int NR>
sb_status rows_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = AtShape<DP, NR>;
    auto* kernel = kv8_rows_kernel<TYPE, DP, NR>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (max_new * a.group + S::ROWS - 1) / S::ROWS;
    const int64_t tiles = row_tiles * a.g.heads * a.g.requests;
    if (tiles >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: too many query rows");
    // a share per resident CTA, fewer if there cannot be so many shares
    int64_t keys = max_len;
    if (a.window > 0 && keys > a.window + S::ROWS + SB_KV8_BLOCK) keys = a.window + S::ROWS + SB_KV8_BLOCK;
    const int64_t steps = (keys + AT_STEP - 1) / AT_STEP + 1;
    // Units of a share at least. A step takes a share about 0.22 us, and every piece of an item 0.22 us per
    // eight rows when they are added: u units a share cost u + steps NR / u. Fixed shares of 6, 16 and
    // 28 took 12, 16 and 18 us for one request in 2000 (8 rows), 43, 35 and 31 for one in 8192 (16 rows).
    a.least = 6;
    while ((int64_t)a.least * a.least < steps * NR) ++a.least;
    const int64_t most = (tiles * (steps + AT_EXTRA) + a.least - 1) / a.least;
    const int64_t ctas = most < (int64_t)S::CTAS * ctx->sm_count ? most : (int64_t)S::CTAS * ctx->sm_count;
    a.row_tiles = (int)row_tiles;
    a.by_row_tiles = KvDiv(a.row_tiles);
    const size_t n = (size_t)ctas * 2 * S::ROWS;
    void* arena;
    const sb_status s = sb_scratch(ctx, Carver::need({n * a.g.dim * 4, n * 8}), &arena);
    if (s != SB_OK) return s;
    Carver cv(arena);
    a.part = cv.take<float>(n * a.g.dim);
    a.part_ml = cv.take<float2>(n);
    if (ctx->kv8_done_n < (size_t)tiles) {
        // Zeroed once; every call leaves zeros.  The old counters stay for captured launches.  They are zeroed here and
        // now, on a stream of their own: in a capture the context's stream would only do it when the graph is replayed.
        const size_t want_n = (size_t)tiles * 2 + 4096;
        unsigned* fresh = nullptr;
        if (cudaMalloc(&fresh, want_n * 4) != cudaSuccess) {
            (void)cudaGetLastError();
            return sb_fail(ctx, SB_ERR_SCRATCH, "kv8 attention: %zu counters", want_n);
        }
        cudaStream_t once = nullptr;
        cudaError_t e = cudaStreamCreateWithFlags(&once, cudaStreamNonBlocking);
        if (e == cudaSuccess) e = cudaMemsetAsync(fresh, 0, want_n * 4, once);
        if (e == cudaSuccess) e = cudaStreamSynchronize(once);
        if (once) cudaStreamDestroy(once);
        if (e != cudaSuccess) {
            (void)cudaGetLastError();
            cudaFree(fresh);
            return sb_fail(ctx, SB_ERR_CUDA, "kv8 attention: zeroing %zu counters: %s", want_n, cudaGetErrorString(e));
        }
        if (ctx->kv8_done) ctx->retired.push_back(ctx->kv8_done);
        ctx->kv8_done = fresh;
        ctx->kv8_done_n = want_n;
    }
    a.done = ctx->kv8_done;
    kernel<<<(unsigned)ctas, AT_WARPS * 32, S::SMEM, ctx->stream>>>(a);
    SB_LAUNCHED(ctx);
    return SB_OK;
}

template <int TYPE, int DP>
sb_status rows_by_count(sb_ctx* ctx, const AtArgs& a, int64_t max_new, int64_t max_len) {
    const int64_t rows = max_new * a.group;
    if (rows <= 8) return rows_launch<TYPE, DP, 1>(ctx, a, max_new, max_len);
    if (rows <= 16 || DP == 256) return rows_launch<TYPE, DP, 2>(ctx, a, max_new, max_len);
    return rows_launch<TYPE, DP, DP == 256 ? 2 : 3>(ctx, a, max_new, max_len);
}
template <int TYPE>
sb_status rows_by_dim(sb_ctx* ctx, const AtArgs& a, int64_t max_new, int64_t max_len) {
    return a.g.dim <= 64 ? rows_by_count<TYPE, 64>(ctx, a, max_new, max_len)
         : a.g.dim <= 128 ? rows_by_count<TYPE, 128>(ctx, a, max_new, max_len) : rows_by_count<TYPE, 256>(ctx, a, max_new, max_len);
}

}  // namespace

extern "C" sb_status sb_kv8_attention(sb_ctx* ctx, const sb_kv8_cache* cache, const void* Q, int64_t q_token_stride,
                                      int64_t q_head_stride, int q_heads, int64_t total, const int32_t* starts,
                                      const int32_t* lens, int64_t max_new, int64_t max_len, float scale, int64_t window,
                                      void* O, int64_t o_token_stride, int64_t o_head_stride, float* lse) {
    if (!ctx) return SB_ERR_INVALID;
    const sb_status s = kv8_check(ctx, "kv8 attention", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!Q || !O) return sb_fail(ctx, SB_ERR_INVALID, "kv8 attention: null");
    if (q_heads <= 0 || q_heads % cache->heads) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: q_heads must be a multiple of the cache's heads");
    if (max_len < 1 || window < 0 || !(scale == scale))
        return sb_fail(ctx, SB_ERR_INVALID, "kv8 attention: max_len below 1, negative window or scale not a number");
    const int64_t most = kv8_table_pages(cache) * cache->page_tokens;
    if (max_len > most) max_len = most;
    if (!kv8_aligned16(Q) || !kv8_aligned16(O) || q_token_stride % 8 || q_head_stride % 8 || o_token_stride % 8 || o_head_stride % 8)
        return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: strides that are multiples of 8 and 16-byte aligned bases");
    if (max_new * (q_heads / cache->heads) >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: max_new x query heads too large");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    AtArgs a{};
    a.g = kv8_geom(cache, total, starts, lens, max_new);
    a.k = static_cast<const uint8_t*>(cache->k); a.v = static_cast<const uint8_t*>(cache->v);
    a.k_scale = static_cast<const uint16_t*>(cache->k_scale); a.v_scale = static_cast<const uint16_t*>(cache->v_scale);
    a.q = static_cast<const __nv_bfloat16*>(Q); a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.o = static_cast<__nv_bfloat16*>(O); a.o_token_stride = o_token_stride; a.o_head_stride = o_head_stride;
    a.lse = lse;
    a.group = q_heads / cache->heads;
    a.by_group = KvDiv(a.group);
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window >= (1ll << 30) ? 0 : (int)window;
    a.st = ctx->dstate;
    // Many query rows per cache head: a key is converted once for 256 rows and the products run at the
    // rate of tcgen05; few: the cache's bytes bound the call and 8 to 24 rows per warp are enough. That kernel's
    // shared memory holds heads of up to 128; wider ones stay here, where every 16 rows read and convert the cache
    // again: 4 requests of up to 1024 tokens behind up to 8192 take 3.3 ms with heads of 256, 255 us with heads of 128.
    if (max_new * a.group > AT_PROMPT_FROM && cache->dim <= 128) return kv8_prompt(ctx, a, cache->type, max_new, max_len);
    return cache->type == SB_KV_INT8 ? rows_by_dim<SB_KV_INT8>(ctx, a, max_new, max_len) : rows_by_dim<SB_KV_E4M3>(ctx, a, max_new, max_len);
}
