// Pieces of the kernels for few query rows (kv8_attention.cu, kv4_attention.cu): instructions, a CTA's share of the work, the
// sum of an item's pieces, the plan of a launch.
#pragma once
#include "kv8_attention.cuh"

namespace {

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

// Where this CTA's share of all items' units starts and how long it is; false: there is none. DIRECT: it has an item of its own.
template <class S, bool DIRECT>
__device__ __forceinline__ bool at_share(const AtArgs& a, unsigned char* smem, AtWalk<S::ROWS, AT_STEP, AT_EXTRA>& wk, long long& share) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (DIRECT) {
        const int row_tile = blockIdx.x / a.g.heads;
        const AtItem it = at_item<S::ROWS, AT_STEP>(a, row_tile);
        share = it.steps + AT_EXTRA;
        return it.steps && wk.begin(a, it, row_tile, (int)blockIdx.x - row_tile * a.g.heads, 0, 0, share);
    }
    // units of one head before each row tile of all requests, 128 at a time
    struct Found {
        AtItem it;
        int row_tile, head, unit;
    };
    long long* sums = reinterpret_cast<long long*>(smem);       // [AT_WARPS] and, behind them, where the share starts
    Found* found = reinterpret_cast<Found*>(sums + AT_WARPS);
    const int n = a.row_tiles * a.g.requests;
    AtItem it;
    auto units = [&](int i) -> long long {
        it.steps = 0;
        if (i < n) it = at_item<S::ROWS, AT_STEP>(a, i);
        return it.steps ? it.steps + AT_EXTRA : 0;
    };
    long long mine = units(threadIdx.x), x = mine, total = 0;
    if (n > AT_WARPS * 32) {
        for (int i = threadIdx.x + AT_WARPS * 32; i < n; i += AT_WARPS * 32) x += units(i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane == 0) sums[warp] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < AT_WARPS; ++w) total += sums[w];
    }
    long long before = 0, at = 0;
    for (int base = 0; base < n; base += AT_WARPS * 32) {
        if (n > AT_WARPS * 32) {
            mine = units(base + threadIdx.x);
            __syncthreads();
        }
        x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        long long all = 0, below = before;
#pragma unroll
        for (int w = 0; w < AT_WARPS; ++w) {
            if (w < warp) below += sums[w];
            all += sums[w];
        }
        if (base == 0) {
            total = (n > AT_WARPS * 32 ? total : all) * a.g.heads;
            share = at_div(total + gridDim.x - 1, gridDim.x);
            if (share < a.least) share = a.least;
            at = blockIdx.x * share;
            if (at >= total) return false;
        }
        const long long lo = (below + x - mine) * a.g.heads;     // the row tile's first unit of all
        if (at >= lo && at < lo + mine * a.g.heads) {
            found->it = it;
            found->row_tile = base + threadIdx.x;
            found->head = (int)at_div(at - lo, mine);
            found->unit = (int)(at - lo - found->head * mine);
        }
        before += all;
        if (at < before * a.g.heads) break;
    }
    __syncthreads();
    const Found f = *found;
    __syncthreads();
    return wk.begin(a, f.it, f.row_tile, f.head, f.unit, at, min(share, total - at));
}

// The warps' sums of a piece (osm [warp][row][OPITCH] and, behind it, their references and sums of weights) become results, or where
// the item has other pieces an entry in scratch; the last piece to finish adds those.
template <class S, int DP, bool DIRECT>
__device__ __forceinline__ void at_finish(const AtArgs& a, unsigned char* smem, const AtWalk<S::ROWS, AT_STEP, AT_EXTRA>& wk, long long share) {
    const int lane = threadIdx.x & 31;
    const int D = a.g.dim, head = wk.head, r0 = wk.it.r0, nrow = wk.it.nrow;
    const Kv8Request rq = wk.it.rq;
    const float* osm = reinterpret_cast<const float*>(smem);
    const float2* mlsm = reinterpret_cast<const float2*>(smem + (size_t)AT_WARPS * S::ROWS * S::OPITCH * 4);
    const bool whole = DIRECT || wk.count == wk.it.steps;
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
            // weights of the pieces of every row in shared memory; a row for as many lanes as there are pieces, up to a warp
            float* weight = reinterpret_cast<float*>(smem);          // [pieces][ROWS]
            float2* total = reinterpret_cast<float2*>(smem + S::F_AT - S::ROWS * 8);         // (reference, sum) of a row
            const int lanes = pieces <= 4 ? 4 : pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32, part = lane & (lanes - 1);
            for (int r0 = 0; r0 < nrow; r0 += AT_WARPS * 32 / lanes) {
                const int r = r0 + (int)threadIdx.x / lanes;
                const bool row = r < nrow;
                constexpr int HELD = 4;                              // of a lane's pieces in registers
                float2 ml[HELD];
                float mm = -INFINITY, sum = 0.f;
#pragma unroll
                for (int i = 0; i < HELD; ++i) {
                    const int x = part + lanes * i;
                    ml[i] = row && x < pieces ? __ldcg(a.part_ml + slot(x) + r) : make_float2(-INFINITY, 0.f);
                }
#pragma unroll
                for (int i = 0; i < HELD; ++i) mm = fmaxf(mm, ml[i].x);
                for (int x = part + lanes * HELD; row && x < pieces; x += lanes) mm = fmaxf(mm, __ldcg(a.part_ml + slot(x) + r).x);
                for (int o = lanes / 2; o > 0; o >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, o));
                auto put = [&](int x, float2 p) {
                    const float f = p.x == -INFINITY ? 0.f : at_exp2(p.x - mm);
                    weight[x * S::ROWS + r] = f;
                    sum = fmaf(p.y, f, sum);
                };
#pragma unroll
                for (int i = 0; i < HELD; ++i)
                    if (row && part + lanes * i < pieces) put(part + lanes * i, ml[i]);
                for (int x = part + lanes * HELD; row && x < pieces; x += lanes) put(x, __ldcg(a.part_ml + slot(x) + r));
                for (int o = lanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (row && part == 0) total[r] = make_float2(mm, sum);
            }
            __syncthreads();
            constexpr int PER = S::ROWS * DP / 4 / (AT_WARPS * 32);  // outputs of a thread, four columns each, at most
            const int outs = nrow * quads;
            if (outs <= AT_WARPS * 32) {
                // few outputs: one a thread, or several threads for one, each a part of the pieces
                const int parts = AT_WARPS * 32 / outs, mine = (int)threadIdx.x / outs, idx = (int)threadIdx.x - mine * outs;
                const int r = idx / quads, d = 4 * (idx - r * quads);
                float4* shared_sum = reinterpret_cast<float4*>(smem + (S::RING - AT_WARPS * 32 * 16));
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (mine < parts) {
                    const int x1 = pieces * (mine + 1) / parts;
                    constexpr int SIDE = 16;                             // loads side by side: their latency is what this takes
                    for (int x0 = pieces * mine / parts; x0 < x1; x0 += SIDE) {
                        float4 y[SIDE];
#pragma unroll
                        for (int i = 0; i < SIDE; ++i) {
                            y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (x0 + i < x1) y[i] = __ldcg(reinterpret_cast<const float4*>(a.part + (slot(x0 + i) + r) * D + d));
                        }
#pragma unroll
                        for (int i = 0; i < SIDE; ++i) {
                            if (x0 + i >= x1) continue;
                            const float f = weight[(x0 + i) * S::ROWS + r];
                            v.x = fmaf(y[i].x, f, v.x); v.y = fmaf(y[i].y, f, v.y); v.z = fmaf(y[i].z, f, v.z); v.w = fmaf(y[i].w, f, v.w);
                        }
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
}

// Rows, shares, scratch and counters of a launch of `ctas` blocks.
template <class S>
sb_status at_rows_plan(sb_ctx* ctx, const char* what, AtArgs& a, int64_t max_new, int64_t max_len, int64_t& ctas) {
    const int64_t row_tiles = (max_new * a.group + S::ROWS - 1) / S::ROWS;
    const int64_t tiles = row_tiles * a.g.heads * a.g.requests;
    if (tiles >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "%s: too many query rows", what);
    // a share per resident CTA, fewer if there cannot be so many shares
    int64_t keys = max_len;
    if (a.window > 0 && keys > (int64_t)a.window + S::ROWS + SB_KV8_BLOCK) keys = (int64_t)a.window + S::ROWS + SB_KV8_BLOCK;
    const int64_t steps = (keys + AT_STEP - 1) / AT_STEP + 1;
    a.row_tiles = (int)row_tiles;
    a.by_row_tiles = KvDiv(a.row_tiles);
    // Short items: a CTA each, without the search for a share, scratch and the sum of pieces. Heads of 128, us, in shares and so, 4 and
    // 8 bits: 22 requests of 20 rows in 70 tokens 13.9 and 7.2, 15.4 and 9.1; 1 of 4 rows and 8 heads in 200 8.7 and 4.6, 9.3 and
    // 5.8; in 500 9.5 and 6.1, 10.2 and 8.0; in 900 9.7 and 9.6, 10.4 and 13.0; 48 in 900 21.9 and 15.6, 25.2 and 19.3; in
    // 1500 28 and 22, 34 and 28; 60 in 1500 (a few items more than fit at once) 32.5 and 32, 40 and 48. Heads of other sizes, 4 rows and 8
    // heads: 1 in 500 of 64 8.5 and 5.2, 9.7 and 7.0, of 80 9.4 and 6.9, 10.5 and 9.2, of 208 11.9 and 10.0, 13.5 and 13.1, of 256 11.9 and
    // 8.6, 12.8 and 11.1; 4 bits, 1 in 1000 of 64 8.9 and 7.5, of 80 9.5 and 10.8, of 208 13.8 and 15.8, of 256 13.8 and 13.3, 48 in 1000
    // 18.6 and 13.6, 25.6 and 18.8, 52.7 and 36.8, 45.7 and 31.2.
    // Not where most of very many CTAs would find nothing (slots without a request's tokens; us in shares and so): heads of 128, 8 cache
    // heads, one of 512 slots in 60 tokens 6.6 and 5.7, 7.7 and 6.0, in 500 11.3 and 6.5, 11.8 and 8.6; one of 1024 in 60 7.9 and 10.3, 9.0
    // and 10.4, in 500 12.7 and 10.4, 13.2 and 10.6; one of 4096 in 60 15.6 and 38, 17 and 37, in 500 20 and 38, 21 and 38.
    a.direct = steps <= S::DIRECT && tiles - at_real(a, S::ROWS, tiles) <= 64 * (int64_t)ctx->sm_count;
    ctas = tiles;
    if (a.direct) return SB_OK;
    // Units of a share at least. A step takes a share about 0.22 us, and every piece of an item 0.22 us per
    // eight rows when they are added: u units a share cost u + steps NR / u. Fixed shares of 6, 16 and
    // 28 took 12, 16 and 18 us for one request in 2000 (8 rows), 43, 35 and 31 for one in 8192 (16 rows).
    a.least = 6;
    while ((int64_t)a.least * a.least < steps * (S::ROWS / 8)) ++a.least;
    const int64_t most = (tiles * (steps + AT_EXTRA) + a.least - 1) / a.least;
    ctas = most < (int64_t)S::CTAS * ctx->sm_count ? most : (int64_t)S::CTAS * ctx->sm_count;
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
            return sb_fail(ctx, SB_ERR_SCRATCH, "%s: %zu counters", what, want_n);
        }
        cudaStream_t once = nullptr;
        cudaError_t e = cudaStreamCreateWithFlags(&once, cudaStreamNonBlocking);
        if (e == cudaSuccess) e = cudaMemsetAsync(fresh, 0, want_n * 4, once);
        if (e == cudaSuccess) e = cudaStreamSynchronize(once);
        if (once) cudaStreamDestroy(once);
        if (e != cudaSuccess) {
            (void)cudaGetLastError();
            cudaFree(fresh);
            return sb_fail(ctx, SB_ERR_CUDA, "%s: zeroing %zu counters: %s", what, want_n, cudaGetErrorString(e));
        }
        if (ctx->kv8_done) ctx->retired.push_back(ctx->kv8_done);
        ctx->kv8_done = fresh;
        ctx->kv8_done_n = want_n;
    }
    a.done = ctx->kv8_done;
    return SB_OK;
}

}  // namespace
