// Attention of a few query rows over the 4-bit cache: decode steps and drafted tokens.
//
// The products are arranged as over the 8-bit cache (kv8_attention.cu): the KEYS on the 16-row side of mma.sync m16n8k16,
//     S^T[key][row] = K Q^T,     O^T[d][row] += V^T P^T,
// the work of all requests in equal shares, a ring of its own for every warp, filled by cp.async. What differs is the
// operands: a code becomes fp16 by one conversion of two, and its block's scale is multiplied in. An e2m1 code has two
// significant bits and an e4m3 scale four, so the product is exact, and so is its range (2^-10 to 2688). The heads'
// scales go into the factor of the scores and into the sums.
//
// Codes go from shared memory into operand registers without a transposition:
//   K: lane (g, t) of the A operand takes 32 consecutive d of its two tokens (16 bytes each): two blocks of 16.
//   V: lane (g, t) takes 16 consecutive d of four tokens, one block each; the codes of two tokens are interleaved (a byte
//      of both tokens' element d is a pair of the A operand of V^T), two instructions for eight codes.
// Row i of the 16-row side is token T(i) = i / 2 + 4 (i odd) of a half of eight: with it, and rows of a tile placed as
// k4_at says, neither load has bank conflicts.
//
// Precision: as kv8_attention.cu, but a weight is held in fp16 relative to 2^-6 of the row's largest so far.
//
// Measured (heads of 128, four query heads per cache head, 8 cache heads): 64 requests in 8192 67 us, 4.3 TB/s: conversions, multiplications
// by the scales and softmax fill 56 % of the issue slots, the copies' rate would allow 43 us; one in 100000 36 us, of which 15
// are the start and the sum of the pieces; 16 x 5 tokens in a window of 4096 (20 rows) 43 us: 255 registers leave two warps a
// scheduler, and their latencies bound it (three CTAs with spilled registers: 55 us).
#include "kv_rows.cuh"
#include "kv4.cuh"
#include "launch.cuh"

namespace {

constexpr float K4_LIMIT = 16384.f;      // 2^AT4_FAR
// More query rows than this per cache head go to the tcgen05 kernel. Four query rows a token; here and there, us: heads of 64, 16
// requests in 2000 tokens, 64 rows 37 and 41, 96 rows 48 and 41, one in 30000 45 and 50, 50 and 50; heads of 128, 32 rows, one in
// 2000 28 and 22, 4 29 and 26, 16 40 and 49, one in 30000 68 and 50; heads of 256, 4 in 2000, 64 rows 42 and 48, 96 rows 49 and
// 49, 16 108 and 97, 157 and 97, one in 30000 108 and 119, 125 and 119. The number of requests would decide too: the limits
// are near where many of them change sides.
__host__ __device__ constexpr int k4_prompt_from(int dim) { return dim <= 64 ? 80 : dim <= 128 ? 24 : 64; }

template <int BYTES>
__device__ __forceinline__ void k4_copy(unsigned dst, const void* src) {
    if (BYTES == 16) at_copy16(dst, src);
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void k4_copy4(unsigned dst, const void* src, bool take) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(take ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t k4_lds32(unsigned a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t k4_lds16(unsigned a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t k4_lds8(unsigned a) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}

template <int DP, int NR>
struct K4Shape {
    static constexpr int STAGES = DP == 256 || NR == 1 ? 2 : 3;
    static constexpr int CTAS = DP == 256 ? 1 : NR == 1 ? 3 : 2;       // resident per SM: registers and the rings decide
    static constexpr int ROW = DP / 2, SROW = DP / 16;               // bytes of a token's codes and scales
    static constexpr int CODES = AT_STEP * ROW, SCALES = AT_STEP * SROW;
    static constexpr int STAGE = 2 * CODES + 2 * SCALES;             // a step: codes of K and V, scales of K and V
    static constexpr int WARP_RING = STAGES * STAGE;
    static constexpr int ROWS = 8 * NR;
    static constexpr int DIRECT = 33;                                // steps of an item that gets a CTA of its own
    static constexpr int OPITCH = DP + 4;                            // floats of a row of a warp's sums
    static constexpr int SUMS = AT_WARPS * ROWS * (OPITCH + 2) * 4, WEIGHTS = CTAS * 160 * ROWS * 4 + AT_WARPS * 32 * 16;
    static constexpr int RING_NEED = AT_WARPS * WARP_RING > SUMS ? AT_WARPS * WARP_RING : SUMS;
    static constexpr int RING = RING_NEED > WEIGHTS ? RING_NEED : WEIGHTS;      // the warps' sums and the weights of an item's pieces go where the ring was
    static constexpr int QPITCH = 2 * DP + 16;                       // bytes of a query row
    static constexpr int Q_AT = RING;
    static constexpr int F_AT = Q_AT + ROWS * QPITCH;                // score factor of a row, fp32
    static constexpr int FLAG_AT = F_AT + ROWS * 4;
    static constexpr int SMEM = FLAG_AT + 64;
    static_assert(QPITCH >= 8 && WARP_RING % 16 == 0 && SMEM <= 227 * 1024, "");
    static constexpr bool QREGS = NR * DP <= 256;                    // query operands stay in registers
};

// Byte of token `row`'s 16-byte piece in a tile of codes. The eight lanes that load K together take the pieces of tokens q and q + 4,
// the sixteen that load V together a piece or two of tokens q .. q + 3.
template <int DP>
__device__ __forceinline__ unsigned k4_at(int row, int piece) {
    if (DP == 64) return (unsigned)((row ^ ((row >> 1) & 2)) * 32 + piece * 16);
    if (DP == 128) return (unsigned)((row ^ ((row >> 2) & 1)) * 64 + ((piece ^ (row & 2)) << 4));
    return (unsigned)(row * 128 + ((piece ^ ((row & 3) << 1) ^ (row & 4)) << 4));
}

// FULL: a head has DP elements, so a token's bytes are known here. DIRECT: a CTA an item.
template <int DP, int NR, bool FULL, bool DIRECT>
__global__ void __launch_bounds__(AT_WARPS * 32, K4Shape<DP, NR>::CTAS)
kv4_rows_kernel(const AtArgs a) {
    using S = K4Shape<DP, NR>;
    constexpr int KS = DP / 16;                    // contraction steps over d
    constexpr int MT = DP / 16;                    // 16-row tiles of O^T
    constexpr int PANELS = DP == 256 ? 2 : 1;      // of 128 d
    constexpr int KW = DP == 64 ? 2 : 4;           // words of codes a lane takes of a token's keys and panel
    constexpr int VW = DP == 64 ? 1 : 2;           // and values
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int D = a.g.dim;
    const int pitch = FULL ? S::ROW : kv4_code_pitch(D), spitch = FULL ? S::SROW : kv4_scale_pitch(D);
    sb_let_next();
    sb_after_previous();
    AtWalk<S::ROWS, AT_STEP, AT_EXTRA> wk;
    long long share;
    if (!at_share<S, DIRECT>(a, smem, wk, share)) return;
    for (bool more = true; more; more = !DIRECT && wk.next(a)) {
        const int head = wk.head, b = wk.it.b, r0 = wk.it.r0, nrow = wk.it.nrow;
        const Kv8Request rq = wk.it.rq;
        const int i0 = a.by_group.quot(r0), i1 = a.by_group.quot(r0 + nrow - 1);
        const int k0 = wk.it.lo + wk.step0 * AT_STEP, k1 = min(wk.it.hi, k0 + wk.count * AT_STEP);
        const int mine = (wk.count - warp + AT_WARPS - 1) / AT_WARPS;   // steps warp, warp + 4, ...

        // the queries are on their way before the chain of table and codes begins
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

        // ---- where this warp's blocks of 16 tokens lie, AT_BATCH steps at a time: lane 2 s + e holds block e of step s; the
        // table's entries are fetched a batch ahead ----
        auto block_key = [&](int batch) { return k0 + (warp + AT_WARPS * (AT_BATCH * batch + (lane >> 1))) * AT_STEP + SB_KV8_BLOCK * (lane & 1); };
        auto load_entry = [&](int batch) -> int {
            const int key = block_key(batch);
            return key < k1 ? a.g.table[(int64_t)b * a.g.table_stride + a.g.page.quot(key)] : 0;
        };
        // the block's first token of all the cache's rows (-1: no such block)
        auto place = [&](int batch, int entry) -> int64_t {
            const int key = block_key(batch);
            if (key >= k1) return -1;
            if (entry < 0 || entry >= a.g.pages) {
                sb_latch(a.st, SB_ERR_INVALID, SBK_KV4);
                return -1;
            }
            return ((int64_t)entry * a.g.heads + head) * a.g.page_tokens + a.g.page.rem(key);
        };
        int entry_next = load_entry(1);
        int64_t at_even = place(0, load_entry(0)), at_odd = -1;      // of even and odd batches

        const unsigned ring = at_smem(smem) + (unsigned)(warp * S::WARP_RING);
        // copies of step j of this warp into its ring
        constexpr int PIECES = DP / 32, TOKS = 32 / PIECES;          // 16-byte pieces of a token; tokens of one instruction
        const int cp_piece = lane % PIECES, cp_tok = lane / PIECES;
        const int cp_off = cp_tok * pitch + cp_piece * 16, sc_off = (lane & (SB_KV8_BLOCK - 1)) * spitch;
        unsigned cp_to[SB_KV8_BLOCK / TOKS];                         // where this lane's pieces of a block go
#pragma unroll
        for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) cp_to[i] = ring + k4_at<DP>(cp_tok + TOKS * i, cp_piece);
        const unsigned sc_to = ring + (unsigned)(2 * S::CODES + lane * S::SROW);
        auto issue = [&](int j) {
            if (j < mine) {
                const int key = k0 + (warp + AT_WARPS * j) * AT_STEP;
                const unsigned dst = (unsigned)((j % S::STAGES) * S::STAGE);
                const int64_t held = (j / AT_BATCH) & 1 ? at_odd : at_even;
                int64_t base[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) base[e] = __shfl_sync(0xffffffffu, held, 2 * (j & (AT_BATCH - 1)) + e);
                const int64_t sat = (lane < SB_KV8_BLOCK ? base[0] : base[1]) * spitch + sc_off;        // a token's scales per lane
                if (FULL && base[0] >= 0 && base[1] >= 0 && key + AT_STEP <= rq.len) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint8_t *kp = a.k + (base[e] * pitch + cp_off), *vp = a.v + (base[e] * pitch + cp_off);
#pragma unroll
                        for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) {
                            // (a block further on the swizzle is the same)
                            const unsigned to = cp_to[i] + dst + (unsigned)(SB_KV8_BLOCK * e * S::ROW);
                            at_copy16(to, kp + TOKS * i * S::ROW);
                            at_copy16(to + S::CODES, vp + TOKS * i * S::ROW);
                        }
                    }
                    k4_copy<S::SROW>(sc_to + dst, a.k_scale4 + sat);
                    k4_copy<S::SROW>(sc_to + dst + S::SCALES, a.v_scale4 + sat);
                } else {
                    // zeros where there is no block, behind the request's end and behind the row's
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) {
                            const int tok = cp_tok + TOKS * i;
                            const bool take = base[e] >= 0 && key + SB_KV8_BLOCK * e + tok < rq.len && cp_piece * 16 < pitch;
                            const int64_t at = base[e] * pitch + cp_off + TOKS * i * pitch;
                            const unsigned to = cp_to[i] + dst + (unsigned)(SB_KV8_BLOCK * e * S::ROW);
                            at_copy16(to, take ? a.k + at : a.k, take);
                            at_copy16(to + S::CODES, take ? a.v + at : a.v, take);
                        }
                    const bool take = (lane < SB_KV8_BLOCK ? base[0] : base[1]) >= 0 && key + lane < rq.len;
#pragma unroll
                    for (int i = 0; i < S::SROW; i += 4) {
                        const bool in = take && i < spitch;
                        k4_copy4(sc_to + dst + i, in ? a.k_scale4 + sat + i : a.k_scale4, in);
                        k4_copy4(sc_to + dst + S::SCALES + i, in ? a.v_scale4 + sat + i : a.v_scale4, in);
                    }
                }
            }
            at_commit();
        };
#pragma unroll
        for (int j = 0; j < S::STAGES - 1; ++j) issue(j);

        // ---- queries: fp16 rows, each scaled by a power of two ----
        const float by_head = a.k_head ? a.k_head[head] : 1.f;
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
            // (never 0, so that what is masked stays -inf)
            if (lane == 0) reinterpret_cast<float*>(smem + S::F_AT)[r] = fmaxf(__fdiv_rn(fabsf(a.scale_log2), up) * by_head, 1e-37f);
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
        // B operand of step s of panel c: d = 128 c + 2 KS' t + 4 s + {0, 1} and {2, 3} of row g, KS' steps a panel
        const unsigned qlane = at_smem(smem) + S::Q_AT + (unsigned)(g * S::QPITCH + 16 * KW * t);
        uint2 qf[S::QREGS ? KS : 1][NR];
        if (S::QREGS) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
                    qf[s][nr] = at_lds64(qlane + (unsigned)(8 * nr * S::QPITCH + 256 * (s / (2 * KW)) + 8 * (s % (2 * KW))));
        }

        float o[MT][NR][4], m[NR][2], l[NR][2];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) o[i][nr][0] = o[i][nr][1] = o[i][nr][2] = o[i][nr][3] = 0.f;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[nr][e] = -INFINITY; l[nr][e] = 0.f; }

        const int tg = (g >> 1) + 4 * (g & 1);                           // T(g)
        for (int j = 0; j < mine; ++j) {
            if ((j & (AT_BATCH - 1)) == 0) {
                const int batch = j / AT_BATCH;
                if (AT_BATCH * (batch + 1) < mine) {
                    const int64_t at = place(batch + 1, entry_next);
                    if (batch & 1) at_even = at;                         // the slot of the batch before this one
                    else at_odd = at;
                    entry_next = load_entry(batch + 2);
                }
            }
            at_wait<S::STAGES - 2>();
            __syncwarp();
            issue(j + S::STAGES - 1);
            const int key = k0 + (warp + AT_WARPS * j) * AT_STEP;
            const unsigned kst = ring + (unsigned)((j % S::STAGES) * S::STAGE), vst = kst + S::CODES;
            const unsigned kss = vst + S::CODES, vss = kss + S::SCALES;
            // scores, in units of log2
            float s[2][NR][4];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) s[e][nr][0] = s[e][nr][1] = s[e][nr][2] = s[e][nr][3] = 0.f;
#pragma unroll
            for (int c = 0; c < PANELS; ++c) {
                // both halves of the step side by side: twice the independent products
                uint32_t w[2][2][KW], sc[2][2][2];                       // [half][token T(g), T(g) + 8]
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = SB_KV8_BLOCK * e + 8 * h + tg;
                        if constexpr (DP == 64) {
                            const uint2 x = at_lds64(kst + k4_at<DP>(row, t >> 1) + 8 * (t & 1));
                            w[e][h][0] = x.x; w[e][h][1] = x.y;
                            const uint32_t s1 = e4m3x2_to_f16x2(k4_lds8(kss + row * S::SROW + t));
                            sc[e][h][0] = __byte_perm(s1, s1, 0x1010);
                        } else {
                            const uint4 x = at_lds128(kst + k4_at<DP>(row, 4 * c + t));
                            w[e][h][0] = x.x; w[e][h][1] = x.y; w[e][h][2] = x.z; w[e][h][3] = x.w;
                            const uint32_t s2 = e4m3x2_to_f16x2(k4_lds16(kss + row * S::SROW + 8 * c + 2 * t));
                            sc[e][h][0] = __byte_perm(s2, s2, 0x1010);
                            sc[e][h][1] = __byte_perm(s2, s2, 0x3232);
                        }
                    }
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    uint32_t p[2][2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            fp4_unpack8(w[e][h][i], p[e][h]);
#pragma unroll
                            for (int k = 0; k < 4; ++k) p[e][h][k] = f16x2_mul(p[e][h][k], sc[e][h][i >> 1]);
                        }
                    uint4 q4[NR];
                    if constexpr (!S::QREGS) {
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) q4[nr] = at_lds128(qlane + (unsigned)(8 * nr * S::QPITCH + 256 * c + 16 * i));
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int nr = 0; nr < NR; ++nr) {
                            uint2 qb;
                            if constexpr (S::QREGS) qb = qf[2 * KW * c + 2 * i + u][nr];
                            else qb = u ? make_uint2(q4[nr].z, q4[nr].w) : make_uint2(q4[nr].x, q4[nr].y);
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                at_mma(s[e][nr], p[e][0][2 * u], p[e][1][2 * u], p[e][0][2 * u + 1], p[e][1][2 * u + 1], qb.x, qb.y);
                        }
                }
            }
            const bool edge = key + AT_STEP > rq.past + i0 + 1 || key + AT_STEP > k1 || (a.window > 0 && key <= rq.past + i1 - a.window);
            if (edge) {
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int kk = key + SB_KV8_BLOCK * e + tg + 8 * (i >> 1), p = pos[nr][i & 1];
                            if (kk > p || kk >= k1 || (a.window > 0 && kk <= p - a.window)) s[e][nr][i] = -INFINITY;
                        }
            }
            // The weights by the reference there is. A lane's sum says whether that still does: no weight is above it. One above 2^AT4_FAR
            // (or none: NaN), or a row's first key, takes the way by the rows' maxima, and the weights anew.
            uint32_t pb[2][NR][2];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float sum[2];
                auto weights = [&]() {
                    sum[0] = sum[1] = 0.f;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float mm = m[nr][i & 1];
                            p[i] = at_exp2(fmaf(s[e][nr][i], fq[nr][i & 1], mm == -INFINITY ? 0.f : -mm));
                            sum[i & 1] += p[i];
                        }
                        pb[e][nr][0] = at_half2(p[0], p[1]);
                        pb[e][nr][1] = at_half2(p[2], p[3]);
                    }
                };
                weights();
                const bool far = !(sum[0] <= K4_LIMIT && sum[1] <= K4_LIMIT) || m[nr][0] == -INFINITY || m[nr][1] == -INFINITY;
                if (__any_sync(0xffffffffu, far)) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(fmaxf(s[0][nr][e], s[0][nr][2 + e]), fmaxf(s[1][nr][e], s[1][nr][2 + e]));
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                        mx *= fq[nr][e];                                 // factors are positive
                        f[e] = 1.f;
                        if (mx > m[nr][e] + AT4_FAR) {
                            const float ref = mx - AT4_UP;
                            f[e] = at_exp2(m[nr][e] - ref);
                            m[nr][e] = ref;
                            l[nr][e] *= f[e];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[i][nr][0] *= f[0]; o[i][nr][1] *= f[1]; o[i][nr][2] *= f[0]; o[i][nr][3] *= f[1];
                    }
                    weights();
                }
                l[nr][0] += sum[0];
                l[nr][1] += sum[1];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) {
                    pb[e][nr][0] = at_transpose(pb[e][nr][0]);
                    pb[e][nr][1] = at_transpose(pb[e][nr][1]);
                }
#pragma unroll
                for (int c = 0; c < PANELS; ++c) {
                    // tokens T(2 t), T(2 t + 1), and eight on
                    uint32_t w[4][VW], sb[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int row = SB_KV8_BLOCK * e + t + 4 * k;
                        if constexpr (DP == 64) {
                            w[k][0] = k4_lds32(vst + k4_at<DP>(row, g >> 2) + 4 * (g & 3));
                            sb[k] = k4_lds8(vss + row * S::SROW + (g >> 1));
                        } else {
                            const uint2 x = at_lds64(vst + k4_at<DP>(row, 4 * c + (g >> 1)) + 8 * (g & 1));
                            w[k][0] = x.x; w[k][1] = x.y;
                            sb[k] = k4_lds8(vss + row * S::SROW + 8 * c + g);
                        }
                    }
                    const uint32_t slo = e4m3x2_to_f16x2(sb[0] | sb[1] << 8), shi = e4m3x2_to_f16x2(sb[2] | sb[3] << 8);
#pragma unroll
                    for (int i = 0; i < VW; ++i) {
                        // even and odd elements of eight, of two tokens side by side
                        constexpr uint32_t LO = 0x0f0f0f0fu;
                        uint32_t el[4], ol[4], eh[4], oh[4];
                        fp4_unpack8((w[0][i] & LO) | (w[1][i] << 4 & ~LO), el);
                        fp4_unpack8((w[0][i] >> 4 & LO) | (w[1][i] & ~LO), ol);
                        fp4_unpack8((w[2][i] & LO) | (w[3][i] << 4 & ~LO), eh);
                        fp4_unpack8((w[2][i] >> 4 & LO) | (w[3][i] & ~LO), oh);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t a0 = f16x2_mul(el[k], slo), a1 = f16x2_mul(ol[k], slo), a2 = f16x2_mul(eh[k], shi), a3 = f16x2_mul(oh[k], shi);
#pragma unroll
                            for (int nr = 0; nr < NR; ++nr) at_mma(o[4 * (VW * c + i) + k][nr], a0, a1, a2, a3, pb[e][nr][0], pb[e][nr][1]);
                        }
                    }
                }
            }
        }
        at_wait<0>();
        __syncthreads();

        // ---- the warps' sums side by side where the ring was ----
        const float back = a.v_head ? a.v_head[head] : 1.f;
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
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    // o[i][.][e] and [2 + e]: two neighbouring d of row r
                    constexpr int LW = DP == 64 ? 8 : 16;                // d a lane holds per panel
                    const int d = LW * g + 128 * (i / (LW / 2)) + 2 * (i % (LW / 2));
                    *reinterpret_cast<float2*>(row + d) = make_float2(o[i][nr][e] * back, o[i][nr][2 + e] * back);
                }
            }
        __syncthreads();
        at_finish<S, DP, DIRECT>(a, smem, wk, share);
        __syncthreads();                                                 // the next piece's copies go where the sums were
    }
}

template <int DP, int NR>
sb_status rows_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = K4Shape<DP, NR>;
    int64_t ctas;
    const sb_status s = at_rows_plan<S>(ctx, "kv4 attention", a, max_new, max_len, ctas);
    if (s != SB_OK) return s;
    auto* kernel = a.direct ? (a.g.dim == DP ? kv4_rows_kernel<DP, NR, true, true> : kv4_rows_kernel<DP, NR, false, true>)
                            : a.g.dim == DP ? kv4_rows_kernel<DP, NR, true, false> : kv4_rows_kernel<DP, NR, false, false>;
    return sb_launch(ctx, kernel, dim3((unsigned)ctas), AT_WARPS * 32, S::SMEM, 1, true, a);
}
template <int DP>
sb_status rows_by_count(sb_ctx* ctx, const AtArgs& a, int64_t max_new, int64_t max_len) {
    const int64_t rows = max_new * a.group;
    if (rows <= 8) return rows_launch<DP, 1>(ctx, a, max_new, max_len);
    if (rows <= 16 || DP == 256) return rows_launch<DP, 2>(ctx, a, max_new, max_len);
    return rows_launch<DP, DP == 256 ? 2 : 3>(ctx, a, max_new, max_len);
}

}  // namespace

extern "C" sb_status sb_kv4_attention(sb_ctx* ctx, const sb_kv4_cache* cache, const void* Q, int64_t q_token_stride,
                                      int64_t q_head_stride, int q_heads, int64_t total, const int32_t* starts,
                                      const int32_t* lens, int64_t max_new, int64_t max_len, float scale, int64_t window,
                                      void* O, int64_t o_token_stride, int64_t o_head_stride, float* lse) {
    if (!ctx) return SB_ERR_INVALID;
    const sb_status s = kv4_check(ctx, "kv4 attention", cache, total, starts, lens, max_new);
    if (s != SB_OK) return s;
    if (total == 0 || max_new == 0) return SB_OK;
    if (!Q || !O) return sb_fail(ctx, SB_ERR_INVALID, "kv4 attention: null");
    if (q_heads <= 0 || q_heads % cache->heads) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 attention: q_heads must be a multiple of the cache's heads");
    if (max_len < 1 || window < 0 || !(scale == scale))
        return sb_fail(ctx, SB_ERR_INVALID, "kv4 attention: max_len below 1, negative window or scale not a number");
    const int64_t most = std::min(kv4_table_pages(cache) * cache->page_tokens, KV_MOST);
    if (max_len > most) max_len = most;
    if (!kv8_aligned16(Q) || !kv8_aligned16(O) || q_token_stride % 8 || q_head_stride % 8 || o_token_stride % 8 || o_head_stride % 8)
        return sb_fail(ctx, SB_ERR_SHAPE, "kv4 attention: strides that are multiples of 8 and 16-byte aligned bases");
    if (max_new * (q_heads / cache->heads) >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv4 attention: max_new x query heads too large");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    AtArgs a{};
    a.g = kv4_geom(cache, total, starts, lens, max_new);
    a.k = static_cast<const uint8_t*>(cache->k); a.v = static_cast<const uint8_t*>(cache->v);
    a.k_scale4 = static_cast<const uint8_t*>(cache->k_scale); a.v_scale4 = static_cast<const uint8_t*>(cache->v_scale);
    a.k_head = cache->k_head; a.v_head = cache->v_head;
    a.q = static_cast<const __nv_bfloat16*>(Q); a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.o = static_cast<__nv_bfloat16*>(O); a.o_token_stride = o_token_stride; a.o_head_stride = o_head_stride;
    a.lse = lse;
    a.group = q_heads / cache->heads;
    a.by_group = KvDiv(a.group);
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window >= KV_MOST ? 0 : (int)window;
    a.st = ctx->dstate;
    if (max_new * a.group > k4_prompt_from(cache->dim)) return kv8_prompt(ctx, a, AT_E2M1, max_new, max_len);
    return cache->dim <= 64 ? rows_by_count<64>(ctx, a, max_new, max_len)
         : cache->dim <= 128 ? rows_by_count<128>(ctx, a, max_new, max_len) : rows_by_count<256>(ctx, a, max_new, max_len);
}
