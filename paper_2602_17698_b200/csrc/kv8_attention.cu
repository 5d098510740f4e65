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
// times its value scale, relative to a running power of two, is rounded to fp16 (2^-11): three
// bits finer than the bf16 result.
//
// Long caches are cut into chunks of keys; a chunk's CTA leaves unnormalised sums, and the last
// CTA of a row tile to finish (a counter) adds the chunks in their order: the result does not
// depend on which one that is.
#include "kv8_attention.cuh"

namespace {

constexpr int AT_PROMPT_FROM = 64;
constexpr int AT_WARPS = 4;
constexpr int AT_STEP = 32;             // keys a warp takes at a time: two scale blocks
constexpr int AT_BATCH = 16;            // steps whose page numbers and scales a warp holds, two lanes a step

__device__ __forceinline__ unsigned at_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
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
    static constexpr int STAGES = DP == 64 ? 4 : 3;
    static constexpr int SIDE = AT_STEP * DP;                      // bytes of a step's keys
    static constexpr int RING = AT_WARPS * STAGES * 2 * SIDE;
    static constexpr int ROWS = 8 * NR;
    static constexpr int QPITCH = 2 * DP + 16;                     // bytes of a query row
    static constexpr int Q_AT = RING;
    static constexpr int F_AT = Q_AT + ROWS * QPITCH;              // score factor of a row, fp32
    static constexpr int FLAG_AT = F_AT + ROWS * 4;
    static constexpr int SMEM = FLAG_AT + 16;
    static constexpr int OPITCH = DP + 4;                          // floats of a row of a warp's sums
    static_assert(AT_WARPS * ROWS * (OPITCH + 2) * 4 <= RING, "the warps' sums fit where the ring was");
    static constexpr bool QREGS = NR * DP <= 256;                  // query operands stay in registers
};

template <int TYPE, int DP, int NR>
__global__ void __launch_bounds__(AT_WARPS * 32)
kv8_rows_kernel(const AtArgs a) {
    using S = AtShape<DP, NR>;
    constexpr int KS = DP / 16;                    // contraction steps over d
    constexpr int MT = DP / 16;                    // 16-row tiles of O^T
    constexpr int PIECES = DP / 16;                // 16-byte pieces of a row
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int split = (int)(blockIdx.x % (unsigned)a.splits), rt = (int)(blockIdx.x / (unsigned)a.splits);
    const int head = blockIdx.y, b = blockIdx.z;
    const int D = a.g.dim;
    Kv8Request rq;
    if (!kv8_request(a.g, b, rq, a.st)) return;
    const int rows = rq.n * a.group, r0 = rt * S::ROWS;
    if (r0 >= rows) return;
    const int nrow = min(S::ROWS, rows - r0);
    // keys that some row of the tile sees, from the start of a scale block
    const int i0 = r0 / a.group, i1 = (r0 + nrow - 1) / a.group;
    const int hi = rq.past + i1 + 1;
    const int lo = a.window > 0 ? max(0, rq.past + i0 - a.window + 1) & ~(SB_KV8_BLOCK - 1) : 0;
    // max_len may be too small: then the chunks grow
    int chunk = a.chunk;
    if ((int64_t)chunk * a.splits < hi - lo) chunk = ((hi - lo + a.splits - 1) / a.splits + AT_STEP - 1) / AT_STEP * AT_STEP;
    const int nsplit = (hi - lo + chunk - 1) / chunk;
    if (split >= nsplit) return;
    const int k0 = lo + split * chunk, k1 = min(hi, k0 + chunk);
    const int nsteps = (k1 - k0 + AT_STEP - 1) / AT_STEP;
    const int mine = (nsteps - warp + AT_WARPS - 1) / AT_WARPS;     // steps warp, warp + 4, ...

    // ---- this warp's page numbers and scales, AT_BATCH steps at a time: lane 2 s + e holds block e of step s ----
    auto block_key = [&](int batch) { return k0 + (warp + AT_WARPS * (AT_BATCH * batch + (lane >> 1))) * AT_STEP + SB_KV8_BLOCK * (lane & 1); };
    auto load_page = [&](int batch) -> int {
        const int key = block_key(batch);
        if (key >= k1) return -1;
        int64_t page;
        return kv8_page(a.g, b, key / a.g.page_tokens, page, a.st) ? (int)page : -1;
    };
    auto load_scales = [&](int batch, int page, uint32_t& s2) {
        s2 = 0;
        if (page < 0) return;
        const int slot = block_key(batch) % a.g.page_tokens;
        const int64_t at = ((int64_t)page * a.g.heads + head) * (a.g.page_tokens / SB_KV8_BLOCK) + slot / SB_KV8_BLOCK;
        s2 = (uint32_t)a.k_scale[at] | (uint32_t)a.v_scale[at] << 16;
    };
    int page_cur = load_page(0), page_next = load_page(1);
    uint32_t sc_cur, sc_next = 0;
    load_scales(0, page_cur, sc_cur);

    const unsigned ring = at_smem(smem) + (unsigned)(warp * S::STAGES * 2 * S::SIDE);
    // copies of step j of this warp into its ring
    auto issue = [&](int j) {
        if (j < mine) {
            const int key = k0 + (warp + AT_WARPS * j) * AT_STEP;
            const unsigned dst = ring + (unsigned)((j % S::STAGES) * 2 * S::SIDE);
            constexpr int TOKS = 32 / (PIECES < 32 ? PIECES : 32);  // tokens a warp copies with one instruction
            const int piece = lane % PIECES, tok_l = lane / PIECES;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int src_lane = 2 * (j & (AT_BATCH - 1)) + e;
                const int pg = __shfl_sync(0xffffffffu, page_cur, src_lane), pgn = __shfl_sync(0xffffffffu, page_next, src_lane);
                const int page = (j / AT_BATCH) & 1 ? pgn : pg;     // page_cur holds even batches, page_next odd ones
                const int slot = (key + SB_KV8_BLOCK * e) % a.g.page_tokens;
                const int64_t base = (((int64_t)max(page, 0) * a.g.heads + head) * a.g.page_tokens + slot) * D;
#pragma unroll
                for (int i = 0; i < SB_KV8_BLOCK / TOKS; ++i) {
                    const int tok = tok_l + TOKS * i;
                    const bool take = page >= 0 && key + SB_KV8_BLOCK * e + tok < rq.len && piece * 16 < D;
                    const int64_t off = take ? base + tok * D + piece * 16 : 0;
                    const int row = SB_KV8_BLOCK * e + tok;
                    const unsigned to = DP == 64 ? (unsigned)(row * 64 + ((piece ^ ((row >> 1) & 3)) << 4))
                                                 : (unsigned)(row * DP + ((piece ^ (row & 7)) << 4));
                    at_copy16(dst + to, a.k + off, take);
                    at_copy16(dst + S::SIDE + to, a.v + off, take);
                }
            }
        }
        at_commit();
    };
#pragma unroll
    for (int j = 0; j < S::STAGES - 1; ++j) issue(j);

    // ---- queries: fp16 rows, each scaled by a power of two ----
    for (int r = warp; r < S::ROWS; r += AT_WARPS) {
        unsigned char* qrow = smem + S::Q_AT + r * S::QPITCH;
        uint32_t w[DP / 64];
        uint32_t amax = 0;
        const int row = r0 + r;
        const __nv_bfloat16* src = a.q + (int64_t)(rq.row0 + row / a.group) * a.q_token_stride +
                                   (int64_t)(head * a.group + row % a.group) * a.q_head_stride;
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) {
            const int d = 64 * i + 2 * lane;
            w[i] = r < nrow && d < D ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
            amax = max(amax, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const float up = at_query_scale(amax);
#pragma unroll
        for (int i = 0; i < DP / 64; ++i)
            *reinterpret_cast<uint32_t*>(qrow + 128 * i + 4 * lane) = at_half2(bf16lo(w[i]) * up, bf16hi(w[i]) * up);
        if (lane == 0) reinterpret_cast<float*>(smem + S::F_AT)[r] = __fdiv_rn(a.scale_log2, up);
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
            pos[nr][e] = rq.past + (r0 + r) / a.group;          // rows past the last: queries of zeros, dropped at the end
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

    float o[MT][NR][4], m[NR][2], l[NR][2];
    float vref = 0.f;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) o[i][nr][0] = o[i][nr][1] = o[i][nr][2] = o[i][nr][3] = 0.f;
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[nr][e] = -INFINITY; l[nr][e] = 0.f; }

    for (int j = 0; j < mine; ++j) {
        if ((j & (AT_BATCH - 1)) == 0) {
            // a new batch: its scales were fetched while the last one ran; fetch the next batch's
            // scales and the page numbers of the one after it (into the slot of the last batch)
            const int batch = j / AT_BATCH;
            if (batch > 0) {
                sc_cur = sc_next;
                if (batch & 1) page_cur = load_page(batch + 1);
                else page_next = load_page(batch + 1);
            }
            if (AT_BATCH * (batch + 1) < mine) load_scales(batch + 1, batch & 1 ? page_cur : page_next, sc_next);
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
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) s[e][nr][0] = s[e][nr][1] = s[e][nr][2] = s[e][nr][3] = 0.f;
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) {
                const int row = SB_KV8_BLOCK * e + g;               // rows g and g + 8 have the same swizzle
                const unsigned off = DP == 64 ? (unsigned)(row * 64 + ((t ^ ((row >> 1) & 3)) << 4))
                                              : (unsigned)(row * DP + 128 * (c >> 1) + (((4 * (c & 1) + t) ^ (row & 7)) << 4));
                const uint4 lo4 = at_lds128(kst + off), hi4 = at_lds128(kst + off + 8 * DP);
                const uint32_t wl[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, wh[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = at_flip<TYPE>(wl[i]), y = at_flip<TYPE>(wh[i]);
                    const uint32_t a0 = at_pair<TYPE, 0>(x), a1 = at_pair<TYPE, 0>(y), a2 = at_pair<TYPE, 1>(x), a3 = at_pair<TYPE, 1>(y);
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) {
                        uint2 qb;
                        if constexpr (S::QREGS) qb = qf[4 * c + i][nr];
                        else qb = at_lds64(qlane + (unsigned)(8 * nr * S::QPITCH + 128 * c + 8 * i));
                        at_mma(s[e][nr], a0, a1, a2, a3, qb.x, qb.y);
                    }
                }
            }
        }
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
            const bool grew = mx[0] > m[nr][0] || mx[1] > m[nr][1];
            if (__any_sync(0xffffffffu, grew)) {
                float f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float mn = fmaxf(m[nr][e], mx[e]);
                    f[e] = mn == -INFINITY ? 1.f : at_exp2(m[nr][e] - mn);
                    m[nr][e] = mn;
                    l[nr][e] *= f[e];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    o[i][nr][0] *= f[0]; o[i][nr][1] *= f[1]; o[i][nr][2] *= f[0]; o[i][nr][3] *= f[1];
                }
            }
        }
        // value scales relative to a power of two that only grows
        const float vmax = fmaxf(vsc[0], vsc[1]);
        if (vmax > vref) {
            const float fresh = at_value_ref(vmax);
            const float f = __fdiv_rn(vref, fresh);
            vref = fresh;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[i][nr][k] *= f;
        }
        const float inv = at_value_inv(vref);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float vw = vsc[e] * inv;
            uint32_t pb[NR][2];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float mm = m[nr][i & 1];
                    p[i] = at_exp2(s[e][nr][i] - (mm == -INFINITY ? 0.f : mm));
                    l[nr][i & 1] += p[i];
                }
                pb[nr][0] = at_transpose(at_half2(p[0] * vw, p[1] * vw));
                pb[nr][1] = at_transpose(at_half2(p[2] * vw, p[3] * vw));
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
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                // o[i][.][e] and [2 + e]: two neighbouring d of row r
                constexpr int LW = DP == 64 ? 8 : 16;                // d a lane holds per panel
                const int d = LW * g + 128 * (i / (LW / 2)) + 2 * (i % (LW / 2));
                *reinterpret_cast<float2*>(row + d) = make_float2(o[i][nr][e] * vref, o[i][nr][2 + e] * vref);
            }
        }
    __syncthreads();
    const int64_t tile = ((int64_t)b * a.g.heads + head) * a.row_tiles + rt;
    auto store = [&](int r, int d, float4 v, float mm, float sum) {
        const int row = r0 + r;
        const int64_t tok = rq.row0 + row / a.group;
        const int h = head * a.group + row % a.group;
        const float f = at_norm(sum);
        const uint2 w = make_uint2(u32(__floats2bfloat162_rn(v.x * f, v.y * f)), u32(__floats2bfloat162_rn(v.z * f, v.w * f)));
        *reinterpret_cast<uint2*>(a.o + tok * a.o_token_stride + h * a.o_head_stride + d) = w;
        if (d == 0 && a.lse) a.lse[tok * (a.g.heads * a.group) + h] = at_lse(mm, sum);
    };
    for (int idx = threadIdx.x; idx < nrow * (D / 4); idx += AT_WARPS * 32) {
        const int r = idx / (D / 4), d = 4 * (idx - r * (D / 4));
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
        if (nsplit == 1) store(r, d, v, mm, sum);
        else {
            const int64_t at = (tile * a.splits + split) * S::ROWS + r;
            *reinterpret_cast<float4*>(a.part + at * D + d) = v;
            if (d == 0) a.part_ml[at] = make_float2(mm, sum);
        }
    }
    if (nsplit == 1) return;
    // ---- the last chunk of the tile to finish adds them all, in order ----
    volatile int* last = reinterpret_cast<volatile int*>(smem + S::FLAG_AT);
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned was = atomicAdd(a.done + tile, 1u);
        *last = was == (unsigned)(nsplit - 1);
        if (*last) a.done[tile] = 0;                                 // for the next call
    }
    __syncthreads();
    if (!*last) return;
    __threadfence();
    for (int idx = threadIdx.x; idx < nrow * (D / 4); idx += AT_WARPS * 32) {
        const int r = idx / (D / 4), d = 4 * (idx - r * (D / 4));
        const int64_t at = tile * a.splits * S::ROWS + r;
        float mm = -INFINITY, sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int x = 0; x < nsplit; ++x) {
            const float2 ml = __ldcg(a.part_ml + at + (int64_t)x * S::ROWS);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part + (at + (int64_t)x * S::ROWS) * D + d));
            const float mn = fmaxf(mm, ml.x);
            const float f = mm == -INFINITY ? 0.f : at_exp2(mm - mn), h = ml.x == -INFINITY ? 0.f : at_exp2(ml.x - mn);
            sum = fmaf(sum, f, ml.y * h);
            v.x = fmaf(v.x, f, y.x * h); v.y = fmaf(v.y, f, y.y * h); v.z = fmaf(v.z, f, y.z * h); v.w = fmaf(v.w, f, y.w * h);
            mm = mn;
        }
        store(r, d, v, mm, sum);
    }
}

template <int TYPE, int DP, int NR>
sb_status rows_launch(sb_ctx* ctx, AtArgs a, int64_t max_new, int64_t max_len) {
    using S = AtShape<DP, NR>;
    auto* kernel = kv8_rows_kernel<TYPE, DP, NR>;
    SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    const int64_t row_tiles = (max_new * a.group + S::ROWS - 1) / S::ROWS;
    // keys a tile can see, and the chunks that make about four CTAs per SM out of all tiles; a chunk
    // is at least eight steps of every warp
    int64_t keys = max_len;
    if (a.window > 0 && keys > a.window + S::ROWS + SB_KV8_BLOCK) keys = a.window + S::ROWS + SB_KV8_BLOCK;
    const int64_t tiles = row_tiles * a.g.heads * a.g.requests;
    const int64_t want = 4 * (int64_t)ctx->sm_count;
    int64_t splits = (want + tiles - 1) / tiles;
    const int64_t least = AT_WARPS * AT_STEP * 4;
    if (splits > (keys + least - 1) / least) splits = (keys + least - 1) / least;
    if (splits < 1) splits = 1;
    a.chunk = (int)(((keys + splits - 1) / splits + AT_STEP - 1) / AT_STEP * AT_STEP);
    a.splits = (int)((keys + a.chunk - 1) / a.chunk);
    a.row_tiles = (int)row_tiles;
    if (row_tiles * a.splits >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "kv8 attention: too many tiles");
    if (a.splits > 1) {
        const size_t n = (size_t)tiles * a.splits * S::ROWS;
        void* arena;
        const sb_status s = sb_scratch(ctx, Carver::need({n * a.g.dim * 4, n * 8}), &arena);
        if (s != SB_OK) return s;
        Carver cv(arena);
        a.part = cv.take<float>(n * a.g.dim);
        a.part_ml = cv.take<float2>(n);
        if (ctx->kv8_done_n < (size_t)tiles) {
            // zeroed once; every call leaves zeros.  The old counters stay for captured launches.
            const size_t want_n = (size_t)tiles * 2 + 4096;
            unsigned* fresh = nullptr;
            if (cudaMalloc(&fresh, want_n * 4) != cudaSuccess) {
                (void)cudaGetLastError();
                return sb_fail(ctx, SB_ERR_SCRATCH, "kv8 attention: %zu counters", want_n);
            }
            SB_CUDA(ctx, cudaMemsetAsync(fresh, 0, want_n * 4, ctx->stream));
            if (ctx->kv8_done) ctx->retired.push_back(ctx->kv8_done);
            ctx->kv8_done = fresh;
            ctx->kv8_done_n = want_n;
        }
        a.done = ctx->kv8_done;
    }
    const dim3 grid((unsigned)(row_tiles * a.splits), (unsigned)a.g.heads, (unsigned)a.g.requests);
    kernel<<<grid, AT_WARPS * 32, S::SMEM, ctx->stream>>>(a);
    SB_LAUNCHED(ctx);
    return SB_OK;
}

template <int TYPE, int DP>
sb_status rows_by_count(sb_ctx* ctx, const AtArgs& a, int64_t max_new, int64_t max_len) {
    const int64_t rows = max_new * a.group;
    return rows <= 8 ? rows_launch<TYPE, DP, 1>(ctx, a, max_new, max_len)
         : rows <= 16 || DP == 256 ? rows_launch<TYPE, DP, 2>(ctx, a, max_new, max_len)
                                   : rows_launch<TYPE, DP, DP == 256 ? 2 : 4>(ctx, a, max_new, max_len);
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
    if (max_len > cache->table_stride * cache->page_tokens) max_len = cache->table_stride * cache->page_tokens;
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
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.window = window >= (1ll << 30) ? 0 : (int)window;
    a.st = ctx->dstate;
    // Many query rows per cache head: a key is converted once for 256 rows and the products run at the
    // rate of tcgen05; few: the cache's bytes bound the call and 8 to 32 rows per warp are enough.
    if (max_new * a.group > AT_PROMPT_FROM && cache->dim <= 128) return kv8_prompt(ctx, a, cache->type, max_new, max_len);
    return cache->type == SB_KV_INT8 ? rows_by_dim<SB_KV_INT8>(ctx, a, max_new, max_len) : rows_by_dim<SB_KV_E4M3>(ctx, a, max_new, max_len);
}
