// What low-rank adapters add to a shared projection: Y = base + scale B (A x), the adapter by request.
//
// Both products run on mma.sync m16n8k16 with rows on the 16-row side: they are a few operations a byte, so the bytes of X, of base
// and Y and of the adapters bound them, and tcgen05 would have little to win.
//
// Few rows a request (decode steps, drafts): one kernel. A cluster of blocks takes a request; each block multiplies its part of `in`,
// adds all parts through distributed shared memory and takes its part of `out`. Operands go from global memory straight into
// registers: the contraction may visit its index in any order, so a lane takes consecutive elements of its operand rows.
//
// Many rows (prompts): two kernels over tiles of 64 rows. The first leaves H = A x in scratch, the blocks of a cluster with a part of
// `in` each; the second adds B H to the base. Both are fed by cp.async through rings in shared memory. The second is launched
// while the first runs and has its first tiles there when that ends. Measured: one token, rank 16, 4096 -> 4096 4.7 us, the chain
// of one launch; 64 tokens of 64 requests, 4096 -> 6144 8.7 us (2.7 TB/s); 6 requests of up to 2048 tokens, rank 64, 4096 -> 6144
// 80 us: 24 for the first product and 56 for the second, where X, base and Y alone are 38. There the pieces of 128 bytes a row
// that a tile of 64 columns makes are part of it (a plain copy in such tiles takes 45), the rest is instructions' latency
// (50 % of issue slots). Tiles of 128 columns, deeper rings, and the second product on tcgen05 came to the same time.
//
// In the second product a lane's columns are made consecutive (column 8 (n / 2) + 2 j + n % 2 is column n of tile j), so base and Y
// move in 16-byte pieces. H is held as the sum of two bf16 numbers, h = hi + lo with lo = bf16(h - hi): what is lost is below 2^-17 of
// h, so the result's one rounding decides.
#include "kv8.cuh"
#include "launch.cuh"

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
    int splits;                  // of `in`: blocks of a cluster
    int64_t columns;             // of a block of the second product, a multiple of its tiles' columns
    uint16_t* h;                 // [2: hi, lo][total][padded rank], bf16
    SbDeviceState* st;
};

__device__ __forceinline__ void lo_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lo_ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

struct LoTile { int64_t row0; int rows, adapter; };
// The rows of a request and its adapter; no rows (and the status latched) where its numbers do not fit. L2: by way of L2, as a kernel
// has to that reads before its own wait. With few rows a block's warps find in L1 what the first has read (64 requests of one row 9.4 us
// and so 8.7); lora_down_kernel was faster by way of L2 (6 x 1500 rows of rank 16 74.7 us and 69.7, both kernels).
template <bool L2>
__device__ __forceinline__ LoTile lo_request(const LoArgs& a, int b) {
    auto number = [](const int32_t* p) -> int { return L2 ? __ldcg(p) : *p; };
    LoTile t;
    t.row0 = number(a.starts + b);
    t.adapter = number(a.ids + b);
    const int64_t n = (int64_t)number(a.starts + b + 1) - t.row0;
    const bool fits = t.row0 >= 0 && n >= 0 && n <= a.max_new && t.row0 + n <= a.total;
    t.rows = fits ? (int)n : 0;
    if (!fits || t.adapter < -1 || t.adapter >= a.adapters) {
        sb_latch(a.st, SB_ERR_INVALID, SBK_LORA);
        t.adapter = -1;
    }
    return t;
}
// Tile number `tile`; all threads of the block take part. rows = 0: there is no such tile.
template <int TM, int THREADS, bool L2>
__device__ __forceinline__ LoTile lo_tile(const LoArgs& a, int tile) {
    if (a.direct) return lo_request<L2>(a, tile);
    __shared__ int sums[THREADS / 32];
    __shared__ LoTile found;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) found.rows = 0;
    int64_t before = 0;                                              // 64 bits: starts that go down may count rows more than once
    for (int base = 0; base < a.requests; base += THREADS) {
        LoTile t{0, 0, -1};
        if (base + threadIdx.x < a.requests) t = lo_request<L2>(a, base + threadIdx.x);
        const int mine = (t.rows + TM - 1) / TM;
        int x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        int64_t all = 0, below = before;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < warp) below += sums[w];
            all += sums[w];
        }
        const int64_t lo = below + x - mine;
        if (tile >= lo && tile < lo + mine) {
            t.row0 += (tile - lo) * TM;
            t.rows = (int)min((int64_t)TM, t.rows - (tile - lo) * TM);
            found = t;
        }
        before += all;
        if (tile < before) break;
    }
    __syncthreads();
    return found;
}

__device__ __forceinline__ unsigned lo_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void lo_copy16(unsigned dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void lo_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void lo_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void lo_ldsm4(unsigned a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint4 lo_lds16(unsigned a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lo_lds8(unsigned a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void lo_cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void lo_cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// four floats of another block's shared memory, where they are `own` in this one
__device__ __forceinline__ float4 lo_peer(const float* own, unsigned rank) {
    unsigned at;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(lo_smem(own)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
// the sum of all blocks' four floats, in the blocks' order, as two pairs of bf16 each: hi and lo
__device__ __forceinline__ void lo_total(const float* own, int blocks, uint2& hi, uint2& lo) {
    float4 v = blocks > 1 ? lo_peer(own, 0) : *reinterpret_cast<const float4*>(own);
    for (int b = 1; b < blocks; ++b) {
        const float4 w = lo_peer(own, b);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    const float f[4] = {v.x, v.y, v.z, v.w};
    uint32_t top[2], rest[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        top[i] = u32(__floats2bfloat162_rn(f[2 * i], f[2 * i + 1]));
        // (of an infinity nothing is left)
        const float x = f[2 * i] - bf16lo(top[i]), y = f[2 * i + 1] - bf16hi(top[i]);
        rest[i] = u32(__floats2bfloat162_rn(fabsf(bf16lo(top[i])) < INFINITY ? x : 0.f, fabsf(bf16hi(top[i])) < INFINITY ? y : 0.f));
    }
    hi = make_uint2(top[0], top[1]);
    lo = make_uint2(rest[0], rest[1]);
}

// ---- Y = base + scale B H ----
template <typename T> struct LoOut;
template <> struct LoOut<__nv_bfloat16> {
    uint4 v;
    // from shared memory: 16 bytes (fp32: and 16 more)
    __device__ __forceinline__ void take(unsigned at, unsigned) { v = lo_lds16(at); }
    // `wide`: the bytes that bases and rows are aligned to, 16 at most
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, int wide) {
        if (wide == 16 && left >= 8) v = *reinterpret_cast<const uint4*>(p);
        else if (wide == 8 && left >= 8) {
            const uint2 x = *reinterpret_cast<const uint2*>(p), y = *reinterpret_cast<const uint2*>(p + 4);
            v = make_uint4(x.x, x.y, y.x, y.y);
        } else if (wide == 4 && left >= 8) {
            const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
            v = make_uint4(q[0], q[1], q[2], q[3]);
        } else {
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
    __device__ __forceinline__ void store(__nv_bfloat16* p, int left, int wide) const {
        if (wide == 16 && left >= 8) *reinterpret_cast<uint4*>(p) = v;
        else if (wide == 8 && left >= 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y);
            *reinterpret_cast<uint2*>(p + 4) = make_uint2(v.z, v.w);
        } else if (wide == 4 && left >= 8) {
            uint32_t* q = reinterpret_cast<uint32_t*>(p);
            q[0] = v.x; q[1] = v.y; q[2] = v.z; q[3] = v.w;
        } else {
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
    __device__ __forceinline__ void take(unsigned at, unsigned more) {
        const uint4 p = lo_lds16(at), q = lo_lds16(more);
        v[0] = __uint_as_float(p.x); v[1] = __uint_as_float(p.y); v[2] = __uint_as_float(p.z); v[3] = __uint_as_float(p.w);
        v[4] = __uint_as_float(q.x); v[5] = __uint_as_float(q.y); v[6] = __uint_as_float(q.z); v[7] = __uint_as_float(q.w);
    }
    __device__ __forceinline__ void load(const float* p, int left, int wide) {
        if (wide == 16 && left >= 8) {
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
    __device__ __forceinline__ void store(float* p, int left, int wide) const {
        if (wide == 16 && left >= 8) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = v[i];
        }
    }
};

// A tile of base, ROWS x COLS from p on, into shared memory by THREADS threads; `at`: place of a 16-byte piece of a row. Not where elements
// are not aligned to 4 bytes.
template <typename T, int BYTES, int ROWS, int COLS, int THREADS, typename At>
__device__ __forceinline__ void lo_copy_pieces(unsigned dst, const T* p, int64_t ld, int rows, int64_t left, int tid, const At& at) {
    constexpr int PT = COLS * (int)sizeof(T) / BYTES, PE = BYTES / (int)sizeof(T);         // pieces of a row, elements of one
#pragma unroll(BYTES == 16 ? ROWS * PT / THREADS : 1)
    for (int i = tid; i < ROWS * PT; i += THREADS) {
        const int row = i / PT, piece = i % PT;
        if (row >= rows || PE * (piece + 1) > left) continue;
        const unsigned to = dst + at(row, piece * BYTES / 16) + (unsigned)(piece * BYTES % 16);
        if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p + row * ld + PE * piece) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(p + row * ld + PE * piece), "n"(BYTES) : "memory");
    }
}
template <typename T, int ROWS, int COLS, int THREADS, typename At>
__device__ __forceinline__ void lo_copy_base(unsigned dst, const T* p, int64_t ld, int rows, int64_t left, int wide, int tid, const At& at) {
    if (wide == 16) lo_copy_pieces<T, 16, ROWS, COLS, THREADS>(dst, p, ld, rows, left, tid, at);
    else if (wide == 8) lo_copy_pieces<T, 8, ROWS, COLS, THREADS>(dst, p, ld, rows, left, tid, at);
    else if (wide == 4) lo_copy_pieces<T, 4, ROWS, COLS, THREADS>(dst, p, ld, rows, left, tid, at);
}

// Rows without an adapter: base as it is, columns c0 to c1.
template <typename T>
__device__ __forceinline__ void lo_pass(const LoArgs& a, const LoTile& tile, int64_t c0, int64_t c1, int wide) {
    const T* base = static_cast<const T*>(a.base) + tile.row0 * a.ld_base;
    T* y = static_cast<T*>(a.y) + tile.row0 * a.ldy;
    if (base == y) return;
    for (int r = threadIdx.x >> 5; r < tile.rows; r += 8)
        for (int64_t c = c0 + 8 * (threadIdx.x & 31); c < c1; c += 256) {
            LoOut<T> v;
            const int left = (int)min((int64_t)8, c1 - c);
            v.load(base + r * a.ld_base + c, left, wide);
            v.store(y + r * a.ldy + c, left, wide);
        }
}
// Place of a 16-byte piece of row `row` of B: the eight lanes that load together take every 2 RP / 64-th piece of two neighbouring rows.
template <int RP>
__device__ __forceinline__ unsigned lm_b_at(int row, int piece) {
    if (RP == 128) piece ^= ((piece >> 3) << 1) ^ (row & 1);
    if (RP == 64) piece ^= row & 1;
    return (unsigned)(row * RP * 2 + piece * 16);
}
// The words (pairs along the rank) of row `row` of B that lane t takes
template <int RP>
__device__ __forceinline__ void lo_words(unsigned at, int row, int t, uint32_t (&v)[RP / 8]) {
    constexpr int KW = RP / 8;
    if constexpr (KW >= 4) {
#pragma unroll
        for (int i = 0; i < KW / 4; ++i) {
            const uint4 x = lo_lds16(at + lm_b_at<RP>(row, KW / 4 * t + i));
            v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
        }
    } else {
        const uint2 x = lo_lds8(at + (unsigned)(row * RP * 2 + 8 * t));
        v[0] = x.x; v[1] = x.y;
    }
}
template <typename T>
__device__ __forceinline__ unsigned lf_base_at(int row, int piece) {
    return (unsigned)(row * 32 * (int)sizeof(T) + ((sizeof(T) == 2 ? piece : piece ^ (row & 1)) << 4));
}

// ---- few rows ----
template <int RP, typename T>
struct LfShape {
    static constexpr int NG = RP > 64 ? RP / 64 : 1, KG = 8 / NG;     // warps along the rank and along `in`
    static constexpr int B = 32 * RP * 2, BASE = 16 * 32 * (int)sizeof(T), STAGE = B + BASE;      // of a warp: 32 columns
    static constexpr int CTAS = RP >= 64 ? 1 : 2;                    // resident per SM
    static constexpr int SUMS = KG * 16 * RP * 4;
    static constexpr int H = 2 * 16 * (RP + 8) * 2;
    static constexpr int FIT = (224 * 1024 / CTAS - SUMS - H) / (8 * STAGE), STAGES = FIT > 4 ? 4 : FIT;
    static_assert(STAGES >= 2, "");
    static constexpr int RING = 8 * STAGES * STAGE;
    static constexpr int SMEM = RING + SUMS + H;
};
// A cluster per request, 8 warps a block. RP: rank rounded up to 16, 32, 64 or 128. Every warp brings the operands of its columns
// through a ring of its own, from the start on: they do not wait for the first product.
template <int RP, typename T>
__global__ void __launch_bounds__(256, LfShape<RP, T>::CTAS)
lora_few_kernel(const LoArgs a, const int wide) {
    using S = LfShape<RP, T>;
    constexpr int NG = S::NG, KG = S::KG, NT = RP / 8 / NG;                       // NT: tiles of 8 of the rank a warp has
    constexpr int U = RP == 16 ? 4 : 2;                                          // units of 32 of `in` whose loads overlap
    constexpr int KS = RP / 16, KW = RP / 8;
    extern __shared__ __align__(128) unsigned char lm_smem[];
    float* lo_sums = reinterpret_cast<float*>(lm_smem + S::RING);    // [KG][16][RP]; then the first is the block's sum
    uint16_t* held = reinterpret_cast<uint16_t*>(lm_smem + S::RING + S::SUMS);     // H: [hi, lo][16][RP + 8]
    sb_let_next();
    sb_after_previous();
    const LoTile tile = lo_tile<16, 256, false>(a, blockIdx.x / a.splits);
    const int rank = blockIdx.x % a.splits;                          // of the block in its cluster
    if (tile.rows <= 0) return;
    const int64_t c0 = min(a.out, rank * a.columns), c1 = min(a.out, c0 + a.columns);
    if (tile.adapter < 0) {
        lo_pass<T>(a, tile, c0, c1, wide);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const T* base = static_cast<const T*>(a.base) + tile.row0 * a.ld_base;
    T* y = static_cast<T*>(a.y) + tile.row0 * a.ldy;
    const __nv_bfloat16* b = a.b + (int64_t)tile.adapter * a.out * a.rank;
    const int64_t first = c0 + 32 * warp;
    const unsigned ring = lo_smem(lm_smem) + (unsigned)(warp * S::STAGES * S::STAGE);
    auto issue = [&](int n) {
        const int64_t c = first + 256 * (int64_t)n;
        const unsigned dst = ring + (unsigned)((n % S::STAGES) * S::STAGE);
        if (c < c1) {
            constexpr int PB = RP / 8;                               // pieces of a row of B
#pragma unroll
            for (int i = 0; i < PB; ++i) {
                const int row = (32 * i + lane) / PB, piece = (32 * i + lane) % PB;
                const bool take = c + row < c1 && 8 * piece < a.rank;
                lo_copy16(dst + lm_b_at<RP>(row, piece), take ? b + (c + row) * a.rank + 8 * piece : a.b, take);
            }
            // base, in pieces as wide as its rows are aligned
            const auto at = [](int row, int piece) { return lf_base_at<T>(row, piece); };
            lo_copy_base<T, 16, 32, 32>(dst + S::B, base + c, a.ld_base, tile.rows, c1 - c, wide, lane, at);
        }
        lo_commit();
    };
#pragma unroll
    for (int n = 0; n < S::STAGES - 1; ++n) issue(n);
    {
        const int ng = warp % NG, kg = warp / NG;
        const int64_t units = (a.in + 31) / 32, parts = (int64_t)a.splits * KG, part = (int64_t)rank * KG + kg;
        const int64_t u0 = units * part / parts, u1 = units * (part + 1) / parts;
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
        const __nv_bfloat16 *x0 = a.x + (tile.row0 + min(g, tile.rows - 1)) * a.ldx + 8 * t, *x1 = a.x + (tile.row0 + min(g + 8, tile.rows - 1)) * a.ldx + 8 * t;
        const __nv_bfloat16* w = a.a + ((int64_t)tile.adapter * a.rank + 8 * NT * ng + g) * a.in + 8 * t;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        for (int64_t u = u0; u < u1; u += U) {
            uint4 p[U], q[U], v[U][NT];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int64_t k = 32 * (u + i);
                const bool in = u + i < u1 && k + 8 * t < a.in;
                p[i] = in && g < tile.rows ? lo_ld16(x0 + k) : zero;
                q[i] = in && g + 8 < tile.rows ? lo_ld16(x1 + k) : zero;
#pragma unroll
                for (int n = 0; n < NT; ++n) v[i][n] = in && 8 * (NT * ng + n) < a.rank ? lo_ld16(w + 8 * n * a.in + k) : zero;
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    lo_mma(acc[n], p[i].x, q[i].x, p[i].y, q[i].y, v[i][n].x, v[i][n].y);
                    lo_mma(acc[n], p[i].z, q[i].z, p[i].w, q[i].w, v[i][n].z, v[i][n].w);
                }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float* s = lo_sums + ((kg * 16 + g) * RP + 8 * (NT * ng + n) + 2 * t);
            *reinterpret_cast<float2*>(s) = make_float2(acc[n][0], acc[n][1]);
            *reinterpret_cast<float2*>(s + 8 * RP) = make_float2(acc[n][2], acc[n][3]);
        }
    }
    __syncthreads();
    for (int i = 4 * threadIdx.x; i < tile.rows * RP; i += 1024) {
        float4 sum = *reinterpret_cast<const float4*>(lo_sums + i);
#pragma unroll
        for (int k = 1; k < KG; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(lo_sums + k * 16 * RP + i);
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
        *reinterpret_cast<float4*>(lo_sums + i) = sum;
    }
    if (a.splits > 1) {
        lo_cluster_arrive();
        lo_cluster_wait();
    } else __syncthreads();
    for (int i = 4 * threadIdx.x; i < 16 * RP; i += 1024) {
        uint2 hi = make_uint2(0, 0), lo = hi;
        // behind the rank there are zeros of A, of which an infinity of X makes NaN: zeros here, which meet zeros of B
        if (i < tile.rows * RP && i % RP < a.rank) lo_total(lo_sums + i, a.splits, hi, lo);
        *reinterpret_cast<uint2*>(held + i / RP * (RP + 8) + i % RP) = hi;
        *reinterpret_cast<uint2*>(held + (16 + i / RP) * (RP + 8) + i % RP) = lo;
    }
    if (a.splits > 1) lo_cluster_arrive();                           // what others hold has been read
    __syncthreads();
    uint32_t h[2][2][KW];                                            // [hi, lo][row g, g + 8]
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(held + (16 * k + g + 8 * e) * (RP + 8) + 2 * KW * t);
#pragma unroll
            for (int i = 0; i < KW; ++i) h[k][e][i] = p[i];
        }
    const float scale = a.scale ? a.scale[tile.adapter] : 1.f;
    int n = 0;
    for (int64_t c = first; c < c1; c += 256, ++n) {
        lo_wait<S::STAGES - 2>();
        __syncwarp();
        issue(n + S::STAGES - 1);
        const unsigned at = ring + (unsigned)((n % S::STAGES) * S::STAGE);
        float acc[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t v[KW];
            lo_words<RP>(at, 8 * (g >> 1) + 2 * j + (g & 1), t, v);         // column n of tile j is c + 8 (n / 2) + 2 j + n % 2
            acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int k = 1; k >= 0; --k)
                    lo_mma(acc[j], h[k][0][2 * s], h[k][1][2 * s], h[k][0][2 * s + 1], h[k][1][2 * s + 1], v[2 * s], v[2 * s + 1]);
        }
        const int64_t col = c + 8 * t;                               // a lane's eight columns
        const int left = (int)min((int64_t)8, c1 - col);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = g + 8 * e;
            if (left <= 0 || r >= tile.rows) continue;
            LoOut<T> o;
            if (wide >= 4 && left == 8) o.take(at + S::B + lf_base_at<T>(r, (int)sizeof(T) / 2 * t), at + S::B + lf_base_at<T>(r, 2 * t + 1));
            else o.load(base + r * a.ld_base + col, left, wide);
            const float x[8] = {acc[0][2 * e], acc[0][2 * e + 1], acc[1][2 * e], acc[1][2 * e + 1],
                                acc[2][2 * e], acc[2][2 * e + 1], acc[3][2 * e], acc[3][2 * e + 1]};
            o.add(x, scale);
            o.store(y + r * a.ldy + col, left, wide);
        }
        __syncwarp();
    }
    lo_wait<0>();
    if (a.splits > 1) lo_cluster_wait();
}

// ---- many rows: H = A x ----
constexpr int LM_ROWS = 64;
template <int RP>
struct LmDown {
    static constexpr int STAGES = 4, X = LM_ROWS * 128, STAGE = X + RP * 128;      // a step: 64 of `in`
    static constexpr int SUMS = (RP == 16 ? 2 : 1) * LM_ROWS * RP * 4;
    static constexpr int SMEM = STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS;
};
// 8 warps: 4 groups of 16 rows; 2 halves of the rank, or where that is 16 of every step.
template <int RP>
__global__ void __launch_bounds__(256)
lora_down_kernel(const LoArgs a) {
    using S = LmDown<RP>;
    constexpr int NT = RP == 16 ? 2 : RP / 16;                        // tiles of 8 of the rank a warp has
    extern __shared__ __align__(128) unsigned char lm_smem[];
    // in this order: what the next kernel reads before this one's end (all but H) is there
    sb_after_previous();
    sb_let_next();
    const LoTile tile = lo_tile<LM_ROWS, 256, true>(a, blockIdx.x / a.splits);
    const int part = blockIdx.x % a.splits;
    if (tile.rows <= 0 || tile.adapter < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rg = warp & 3, half = warp >> 2;
    const int64_t steps = (a.in + 63) / 64, s0 = steps * part / a.splits;
    const int mine = (int)(steps * (part + 1) / a.splits - s0);
    const unsigned ring = lo_smem(lm_smem);
    // copies: 16-byte pieces XOR-ed with the row, eight lanes a row
    const int row = threadIdx.x >> 3, piece = threadIdx.x & 7;
    const __nv_bfloat16* x = a.x + tile.row0 * a.ldx + 8 * piece;
    const __nv_bfloat16* w = a.a + (int64_t)tile.adapter * a.rank * a.in + 8 * piece;
    auto issue = [&](int s) {
        if (s < mine) {
            const unsigned dst = ring + (unsigned)((s % S::STAGES) * S::STAGE + (piece ^ (row & 7)) * 16);
            const int64_t k = 64 * (s0 + s);
            const bool in = k + 8 * piece < a.in;
#pragma unroll
            for (int i = 0; i < LM_ROWS; i += 32) {
                const bool take = in && row + i < tile.rows;
                lo_copy16(dst + (unsigned)((row + i) * 128), take ? x + (row + i) * a.ldx + k : a.x, take);
            }
#pragma unroll
            for (int i = 0; i < RP; i += 32) {
                if (RP < 32 && row >= RP) break;
                const bool take = in && row + i < a.rank;
                lo_copy16(dst + S::X + (unsigned)((row + i) * 128), take ? w + (row + i) * a.in + k : a.a, take);
            }
        }
        lo_commit();
    };
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) issue(s);
    const int xr = 16 * rg + (lane & 15), wr = (RP == 16 ? 0 : RP / 2 * half) + (lane & 7) + ((lane >> 4) << 3);
    for (int s = 0; s < mine; ++s) {
        lo_wait<S::STAGES - 2>();
        __syncthreads();
        issue(s + S::STAGES - 1);
        const unsigned at = ring + (unsigned)((s % S::STAGES) * S::STAGE);
#pragma unroll
        for (int k = 0; k < (RP == 16 ? 2 : 4); ++k) {
            const int ks = RP == 16 ? 2 * half + k : k;
            uint32_t xa[4];
            lo_ldsm4(at + (unsigned)(xr * 128 + (((2 * ks + (lane >> 4)) ^ (xr & 7)) << 4)), xa);
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t wb[4];
                lo_ldsm4(at + S::X + (unsigned)((wr + 8 * n) * 128 + (((2 * ks + ((lane >> 3) & 1)) ^ (wr & 7)) << 4)), wb);
                lo_mma(acc[n], xa[0], xa[1], xa[2], xa[3], wb[0], wb[1]);
                lo_mma(acc[n + 1], xa[0], xa[1], xa[2], xa[3], wb[2], wb[3]);
            }
        }
    }
    lo_wait<0>();
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lm_smem);                 // [64][RP] (twice where the halves are of the steps)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float* s = sums + ((RP == 16 ? LM_ROWS * half : 0) + 16 * rg + g) * RP + (RP == 16 ? 0 : RP / 2 * half) + 8 * n + 2 * t;
        *reinterpret_cast<float2*>(s) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(s + 8 * RP) = make_float2(acc[n][2], acc[n][3]);
    }
    __syncthreads();
    if (RP == 16) {
        for (int i = threadIdx.x; i < LM_ROWS * RP; i += 256) sums[i] += sums[LM_ROWS * RP + i];
        __syncthreads();
    }
    if (a.splits > 1) {
        lo_cluster_arrive();
        lo_cluster_wait();
    }
    // a part of the rows for every block
    const int r0 = tile.rows * part / a.splits, r1 = tile.rows * (part + 1) / a.splits;
    for (int i = r0 * RP + 4 * threadIdx.x; i < r1 * RP; i += 1024) {
        uint2 hi = make_uint2(0, 0), lo = hi;
        if (i % RP < a.rank) lo_total(sums + i, a.splits, hi, lo);       // (as in lora_few_kernel)
        uint16_t* h = a.h + tile.row0 * RP + i;
        *reinterpret_cast<uint2*>(h) = hi;
        *reinterpret_cast<uint2*>(h + a.total * RP) = lo;
    }
    if (a.splits > 1) {
        lo_cluster_arrive();
        lo_cluster_wait();
    }
}

// ---- many rows: Y = base + scale B H ----
constexpr int LM_COLS = 64;
template <int RP, typename T>
struct LmUp {
    static constexpr int B = LM_COLS * RP * 2, BASE = LM_ROWS * LM_COLS * (int)sizeof(T), STAGE = B + BASE;
    static constexpr int STAGES = RP == 64 || STAGE > 16384 ? 3 : 4;
    static constexpr int CTAS = RP == 64 ? 3 : 2;                    // at rank 64, 80 registers and three blocks a multiprocessor: 6 x 2048 rows 69 us -> 64
    static constexpr int SMEM = STAGES * STAGE;
};
template <typename T>
__device__ __forceinline__ unsigned lm_base_at(int row, int piece) {
    return (unsigned)(row * LM_COLS * (int)sizeof(T) + ((piece ^ (sizeof(T) == 2 ? (row & 1) << 2 : row & 1)) << 4));
}
// 8 warps: 4 groups of 16 rows, 2 of 32 columns.
template <int RP, typename T>
__global__ void __launch_bounds__(256, LmUp<RP, T>::CTAS)
lora_up_kernel(const LoArgs a, const int wide) {
    using S = LmUp<RP, T>;
    constexpr int KS = RP / 16, KW = RP / 8;
    extern __shared__ __align__(128) unsigned char lm_smem[];
    // starts, ids, B and base are read before this kernel's own wait: lora_down_kernel, which lets it in, has waited for whoever wrote
    // them. They come by way of L2 (.cg); base in narrower pieces can only be copied by way of L1, and waits.
    if (wide < 16) sb_after_previous();
    const LoTile tile = lo_tile<LM_ROWS, 256, true>(a, blockIdx.x);
    const int64_t c0 = (int64_t)blockIdx.y * a.columns, c1 = min(a.out, c0 + a.columns);
    if (tile.rows <= 0 || tile.adapter < 0) {
        sb_after_previous();
        if (tile.rows > 0) lo_pass<T>(a, tile, c0, c1, wide);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rg = warp & 3, cg = warp >> 2;
    const T* base = static_cast<const T*>(a.base) + tile.row0 * a.ld_base;
    T* y = static_cast<T*>(a.y) + tile.row0 * a.ldy;
    const __nv_bfloat16* w = a.b + (int64_t)tile.adapter * a.out * a.rank;
    const int tiles = (int)((c1 - c0 + LM_COLS - 1) / LM_COLS);
    const unsigned ring = lo_smem(lm_smem);
    auto issue = [&](int n) {
        if (n < tiles) {
            const unsigned dst = ring + (unsigned)((n % S::STAGES) * S::STAGE);
            const int64_t c = c0 + LM_COLS * n;
            constexpr int PB = RP / 8;                               // pieces of a row of B
#pragma unroll
            for (int i = 0; i < LM_COLS * PB; i += 256) {
                const int row = (i + (int)threadIdx.x) / PB, piece = (i + (int)threadIdx.x) % PB;
                if (LM_COLS * PB < 256 && row >= LM_COLS) break;
                const bool take = c + row < c1 && 8 * piece < a.rank;
                lo_copy16(dst + lm_b_at<RP>(row, piece), take ? w + (c + row) * a.rank + 8 * piece : a.b, take);
            }
            const auto place = [](int row, int piece) { return lm_base_at<T>(row, piece); };
            lo_copy_base<T, LM_ROWS, LM_COLS, 256>(dst + S::B, base + c, a.ld_base, tile.rows, c1 - c, wide, threadIdx.x, place);
        }
        lo_commit();
    };
#pragma unroll
    for (int n = 0; n < S::STAGES - 1; ++n) issue(n);
    sb_after_previous();                                             // H is there from here on
    uint32_t h[2][2][KW];                                            // [hi, lo][row g, g + 8]
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 16 * rg + g + 8 * e;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(a.h + (k * a.total + tile.row0 + min(r, tile.rows - 1)) * RP + 2 * KW * t);
#pragma unroll
            for (int i = 0; i < KW; i += 2) {
                const uint2 x = __ldcg(reinterpret_cast<const uint2*>(p + i));
                h[k][e][i] = r < tile.rows ? x.x : 0u;
                h[k][e][i + 1] = r < tile.rows ? x.y : 0u;
            }
        }
    const float scale = a.scale ? a.scale[tile.adapter] : 1.f;
    for (int n = 0; n < tiles; ++n) {
        lo_wait<S::STAGES - 2>();
        __syncthreads();
        issue(n + S::STAGES - 1);
        const unsigned at = ring + (unsigned)((n % S::STAGES) * S::STAGE);
        float acc[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = 32 * cg + 8 * (g >> 1) + 2 * j + (g & 1);                // column n of tile j: 8 (n / 2) + 2 j + n % 2
            uint32_t v[KW];
            lo_words<RP>(at, row, t, v);
            acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int k = 1; k >= 0; --k)
                    lo_mma(acc[j], h[k][0][2 * s], h[k][1][2 * s], h[k][0][2 * s + 1], h[k][1][2 * s + 1], v[2 * s], v[2 * s + 1]);
        }
        const int64_t col = c0 + LM_COLS * n + 32 * cg + 8 * t;      // a lane's eight columns
        const int left = (int)min((int64_t)8, c1 - col);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 16 * rg + g + 8 * e;
            if (left <= 0 || r >= tile.rows) continue;
            LoOut<T> o;
            if (wide >= 4 && left == 8)
                o.take(at + S::B + lm_base_at<T>(r, (int)sizeof(T) / 2 * (4 * cg + t)), at + S::B + lm_base_at<T>(r, (int)sizeof(T) / 2 * (4 * cg + t) + 1));
            else o.load(base + r * a.ld_base + col, left, wide);
            const float x[8] = {acc[0][2 * e], acc[0][2 * e + 1], acc[1][2 * e], acc[1][2 * e + 1],
                                acc[2][2 * e], acc[2][2 * e + 1], acc[3][2 * e], acc[3][2 * e + 1]};
            o.add(x, scale);
            o.store(y + r * a.ldy + col, left, wide);
        }
    }
    lo_wait<0>();
}

template <int RP, typename T>
sb_status lo_run(sb_ctx* ctx, LoArgs& a, int wide) {
    a.direct = a.max_new <= 16;
    auto cut = [](int64_t x, int64_t most) { return x < 1 ? 1 : x > most ? most : x; };
    if (a.direct) {
        // blocks of a cluster, a power of two: as many as are resident at once, but 512 of `in` and of `out` each at least
        int64_t want = cut(LfShape<RP, T>::CTAS * ctx->sm_count / a.requests, 16), most = cut((a.in + a.out + 1023) / 1024, 16);
        if (want > most) want = most;
        for (a.splits = 1; 2 * a.splits <= want;) a.splits *= 2;
        a.columns = ((a.out + a.splits - 1) / a.splits + 255) / 256 * 256;
        return sb_launch(ctx, lora_few_kernel<RP, T>, dim3((unsigned)(a.requests * a.splits)), 256, LfShape<RP, T>::SMEM, a.splits, true, a, wide);
    }
    // Tiles that there can be (each has a row at least), and those that there are about: full ones, or one a request where that is more. Parts by
    // full ones alone, and tiles for slots without rows: 127 single rows and one request of 17, rank 16, 85 us, so 47; 64 rows in 20000
    // slots 325 ms and 0.23.
    const int64_t rows = (a.total + LM_ROWS - 1) / LM_ROWS, tiles = std::min(rows + a.requests, a.total);
    const int64_t full = std::max(rows, std::min<int64_t>(a.requests, a.total));
    // parts of `in`: four blocks a multiprocessor, but 256 each at least
    int64_t want = cut(4 * ctx->sm_count / full, 16), most = cut((a.in + 255) / 256, 16);
    if (want > most) want = most;
    for (a.splits = 1; 2 * a.splits <= want;) a.splits *= 2;
    if (tiles * a.splits >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "lora: too many rows");
    const size_t n = (size_t)a.total * RP;
    void* arena;
    sb_status s = sb_scratch(ctx, Carver::need({2 * n * 2}), &arena);
    if (s != SB_OK) return s;
    a.h = Carver(arena).take<uint16_t>(2 * n);
    s = sb_launch(ctx, lora_down_kernel<RP>, dim3((unsigned)(tiles * a.splits)), 256, LmDown<RP>::SMEM, a.splits, true, a);
    if (s != SB_OK) return s;
    // Columns of a block of the second kernel: six or eight blocks a multiprocessor, four tiles each at least; with few rows, one block a
    // multiprocessor of one tile each at least (2 tiles of rows, 144 columns, f32: 17 us in one part, 9.5 in three).
    const int64_t each = (a.out + LM_COLS - 1) / LM_COLS, long_parts = cut((RP == 64 ? 6 : 8) * ctx->sm_count / full, (each + 3) / 4);
    const int64_t short_parts = cut(ctx->sm_count / full, each);
    const int64_t parts = cut(long_parts > short_parts ? long_parts : short_parts, 65535);
    a.columns = (each + parts - 1) / parts * LM_COLS;
    return sb_launch(ctx, lora_up_kernel<RP, T>, dim3((unsigned)tiles, (unsigned)((a.out + a.columns - 1) / a.columns)), 256, LmUp<RP, T>::SMEM, 1, true, a, wide);
}
template <int RP>
sb_status lo_by_type(sb_ctx* ctx, LoArgs& a, int f32, int wide) {
    return f32 ? lo_run<RP, float>(ctx, a, wide) : lo_run<RP, __nv_bfloat16>(ctx, a, wide);
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
    if (Y == X) return sb_fail(ctx, SB_ERR_INVALID, "lora: Y is X");
    if (Y == base && total > 1 && ldy != ld_base) return sb_fail(ctx, SB_ERR_SHAPE, "lora: in place with another leading dimension");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    LoArgs a{};
    a.x = static_cast<const __nv_bfloat16*>(X); a.a = static_cast<const __nv_bfloat16*>(ad->a); a.b = static_cast<const __nv_bfloat16*>(ad->b);
    a.scale = ad->scale; a.base = base; a.y = Y;
    a.ldx = ldx; a.ld_base = ld_base; a.ldy = ldy; a.in = ad->in; a.out = ad->out; a.total = total;
    a.starts = starts; a.ids = ids; a.requests = requests; a.adapters = ad->adapters; a.rank = ad->rank;
    a.max_new = (int)max_new; a.st = ctx->dstate;
    uintptr_t bits = ends | 16;
    if (total > 1) bits |= (uintptr_t)((ld_base | ldy) * size);
    const int wide = (int)(bits & (~bits + 1));
    return ad->rank <= 16 ? lo_by_type<16>(ctx, a, f32, wide) : ad->rank <= 32 ? lo_by_type<32>(ctx, a, f32, wide)
         : ad->rank <= 64 ? lo_by_type<64>(ctx, a, f32, wide) : lo_by_type<128>(ctx, a, f32, wide);
}
