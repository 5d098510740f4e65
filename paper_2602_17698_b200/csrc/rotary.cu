// Rotary positions: pairs of a head's elements turned by an angle that grows with the position.
//
// A block takes a few rows (tokens). It finds their positions, computes cos and sin of rows x rotated / 2 angles once, into
// shared memory, and turns all heads of all parts (queries and keys) with them; a thread takes up to 16 bytes of each half of a
// head ("half") or 16 bytes of neighbouring pairs, one read and one write an element. An angle is position times frequency in 64
// bits, with the product's rounding error by fma, less a multiple of pi / 2 in two parts (Cody and Waite): exact to fp32 for every
// 32-bit position. The bytes bound large calls, the chain of dependent reads small ones.
#include "kv8.cuh"
#include "launch.cuh"

namespace {

constexpr int RO_THREADS = 256;
constexpr int RO_TABLE = 4096;               // angles of a block at most: 32 KB

struct RoPart {
    const void* x;
    void* y;
    int64_t xt, xh, yt, yh;                  // strides, in elements
    int heads;
};
struct RoArgs {
    RoPart part[2];
    const float* freq;
    const int32_t *positions, *starts, *lens;
    int64_t total;
    int requests, max_new;
    int heads, rotated, dim;                 // heads of both parts
    int rows;                                // of a block
    int slots;                               // of a head: pieces that one thread takes
    KvDiv by_slots, by_heads;
    float factor;
    int back;
    SbDeviceState* st;
};

// cos and sin of p * f
__device__ __forceinline__ float2 ro_turn(int p, float f, float factor, bool back) {
    const double x = (double)p, y = (double)f, a = x * y;
    const double n = rint(a * 0.63661977236758134308);               // 2 / pi
    double r = fma(-n, 1.57079632679489655800, a);                   // pi / 2 as a sum of two
    r += fma(x, y, -a) - n * 6.12323399573676603587e-17;
    float s, c;
    sincosf((float)r, &s, &c);
    const long long q = (long long)n;
    if (q & 1) {
        const float t = s;
        s = c;
        c = -t;
    }
    if (q & 2) {
        s = -s;
        c = -c;
    }
    return make_float2(c * factor, (back ? -s : s) * factor);
}

template <typename T, int N> struct alignas(sizeof(T) * N) RoVec { T v[N]; };
__device__ __forceinline__ float ro_float(float x) { return x; }
__device__ __forceinline__ float ro_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T ro_round(float x);
template <> __device__ __forceinline__ float ro_round<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 ro_round<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N: elements of an access. INTER: neighbouring pairs, N / 2 of them an access.
template <typename T, int N, bool INTER>
__global__ void __launch_bounds__(RO_THREADS)
rotary_kernel(const RoArgs a) {
    extern __shared__ __align__(16) unsigned char ro_smem[];
    sb_let_next();
    sb_after_previous();
    const int half = a.rotated / 2;
    float2* table = reinterpret_cast<float2*>(ro_smem);              // [rows][half]
    int* pos = reinterpret_cast<int*>(ro_smem + (size_t)a.rows * half * 8);      // [rows], and whether there is one
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = (int)min((int64_t)a.rows, a.total - row0);
    const int tid = threadIdx.x;
    if (a.positions) {
        for (int i = tid; i < rows; i += RO_THREADS) {
            pos[i] = a.positions[row0 + i];
            pos[a.rows + i] = 1;
        }
    } else {
        for (int i = tid; i < rows; i += RO_THREADS) pos[a.rows + i] = 0;
        auto fits = [&](int64_t s, int64_t n, int len) { return s >= 0 && n >= 0 && n <= a.max_new && s + n <= a.total && len >= n; };
        // every request is looked at by one block for whether it fits
        for (int64_t b = row0 / a.rows * RO_THREADS + tid; b < a.requests; b += (int64_t)gridDim.x * RO_THREADS) {
            const int64_t s = a.starts[b];
            if (!fits(s, a.starts[b + 1] - s, a.lens[b])) sb_latch(a.st, SB_ERR_INVALID, SBK_ROTARY);
        }
        // the requests that may hold these rows: the first from the last start at or before row0 on, by parts of 256
        int64_t lo = 0, hi = a.requests;
        while (hi - lo > RO_THREADS) {
            const int64_t step = (hi - lo + RO_THREADS - 1) / RO_THREADS, at = lo + tid * step;
            const bool in = at < hi;
            const int64_t s = in ? a.starts[at] : 0;
            const int before = __syncthreads_count(in && s <= row0), within = __syncthreads_count(in && s < row0 + rows);
            const int64_t from = lo + max(before - 1, 0) * step, upto = min(hi, lo + within * step);
            if (from == lo && upto == hi) break;
            lo = from;
            hi = upto;
        }
        __syncthreads();
        for (int64_t b = lo + tid; b < hi; b += RO_THREADS) {
            const int64_t s = a.starts[b], n = a.starts[b + 1] - s;
            if (s >= row0 + rows || s + n <= row0) continue;
            const int len = a.lens[b];
            if (!fits(s, n, len)) continue;
            for (int64_t i = max(s, row0); i < min(s + n, row0 + rows); ++i) {
                pos[i - row0] = (int)(len - n + (i - s));
                pos[a.rows + (i - row0)] = 1;
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < rows * half; i += RO_THREADS) {
        const int r = i / half;
        table[i] = ro_turn(pos[a.rows + r] ? pos[r] : 0, __ldg(a.freq + (i - r * half)), a.factor, a.back);
    }
    __syncthreads();
    using V = RoVec<T, N>;
    const int units = rows * a.heads * a.slots;
    for (int u = tid; u < units; u += RO_THREADS) {
        const int rh = a.by_slots.quot(u), slot = u - rh * a.slots, r = a.by_heads.quot(rh);
        int h = rh - r * a.heads;
        if (!pos[a.rows + r]) continue;
        const int k = h >= a.part[0].heads;
        const RoPart& p = a.part[k];
        if (k) h -= a.part[0].heads;
        const T* x = static_cast<const T*>(p.x) + (row0 + r) * p.xt + (int64_t)h * p.xh;
        T* y = static_cast<T*>(p.y) + (row0 + r) * p.yt + (int64_t)h * p.yh;
        const float2* turn = table + r * half;
        if (INTER) {
            constexpr int NP = N / 2 > 0 ? N / 2 : 1;                // N = 1: the two of a pair one by one
            if (N == 1) {
                const int d = 2 * slot;
                const T u0 = x[d], w0 = x[d + 1];
                if (d < a.rotated) {
                    const float2 cs = turn[slot];
                    const float uu = ro_float(u0), ww = ro_float(w0);
                    y[d] = ro_round<T>(uu * cs.x - ww * cs.y);
                    y[d + 1] = ro_round<T>(ww * cs.x + uu * cs.y);
                } else if (x != y) {
                    y[d] = u0;
                    y[d + 1] = w0;
                }
                continue;
            }
            const int d = N * slot;
            if (d >= a.rotated && x == y) continue;
            V v = *reinterpret_cast<const V*>(x + d);
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (d + 2 * i < a.rotated) {
                    const float2 cs = turn[d / 2 + i];
                    const float uu = ro_float(v.v[2 * i]), ww = ro_float(v.v[(2 * i + 1) % N]);
                    v.v[2 * i] = ro_round<T>(uu * cs.x - ww * cs.y);
                    v.v[(2 * i + 1) % N] = ro_round<T>(ww * cs.x + uu * cs.y);
                }
            *reinterpret_cast<V*>(y + d) = v;
        } else if (slot * N < half) {
            const int d = slot * N;
            V v = *reinterpret_cast<const V*>(x + d), w = *reinterpret_cast<const V*>(x + half + d);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float2 cs = turn[d + i];
                const float uu = ro_float(v.v[i]), ww = ro_float(w.v[i]);
                v.v[i] = ro_round<T>(uu * cs.x - ww * cs.y);
                w.v[i] = ro_round<T>(ww * cs.x + uu * cs.y);
            }
            *reinterpret_cast<V*>(y + d) = v;
            *reinterpret_cast<V*>(y + half + d) = w;
        } else {
            const int d = a.rotated + slot * N - half;
            if (x != y) *reinterpret_cast<V*>(y + d) = *reinterpret_cast<const V*>(x + d);
        }
    }
}

template <typename T, int N, bool INTER>
sb_status ro_launch(sb_ctx* ctx, const RoArgs& a) {
    const size_t smem = (size_t)a.rows * (a.rotated / 2) * 8 + (size_t)a.rows * 8;
    return sb_launch(ctx, rotary_kernel<T, N, INTER>, dim3((unsigned)((a.total + a.rows - 1) / a.rows)), RO_THREADS, (int)smem, 1, true, a);
}

}  // namespace

extern "C" sb_status sb_rotary(sb_ctx* ctx, const sb_rotary_table* table, const sb_rotary_part* parts, int n_parts, int dim, int f32,
                               int64_t total, const int32_t* positions, const int32_t* starts, const int32_t* lens, int requests,
                               int64_t max_new) {
    if (!ctx) return SB_ERR_INVALID;
    if (!table || !table->freq || !parts) return sb_fail(ctx, SB_ERR_INVALID, "rotary: null");
    if (n_parts < 1 || n_parts > 2 || total < 0 || max_new < 0 || (f32 != 0 && f32 != 1)) return sb_fail(ctx, SB_ERR_INVALID, "rotary: one or two parts, no negative sizes");
    if (total == 0) return SB_OK;
    if (!positions && (!starts || !lens || requests < 0)) return sb_fail(ctx, SB_ERR_INVALID, "rotary: positions, or starts and lens");
    if (dim < 2 || dim > 1024 || dim % 2 || table->rotated < 2 || table->rotated > dim || table->rotated % 2)
        return sb_fail(ctx, SB_ERR_SHAPE, "rotary: dim even, 2 .. 1024, and rotated even, 2 .. dim");
    if ((table->interleaved | table->inverse) & ~1) return sb_fail(ctx, SB_ERR_INVALID, "rotary: interleaved and inverse are 0 or 1");
    if (!(table->factor - table->factor == 0.f)) return sb_fail(ctx, SB_ERR_INVALID, "rotary: a factor that is not finite");
    if (total >= (1ll << 31) || max_new >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "rotary: at most 2^31 rows");
    if (!positions && requests == 0) return SB_OK;
    RoArgs a{};
    // the widest access that strides, bases and the pairs' places allow
    const int size = f32 ? 4 : 2;
    uintptr_t bits = 0;
    for (int i = 0; i < n_parts; ++i) {
        const sb_rotary_part& p = parts[i];
        if (!p.x || !p.y) return sb_fail(ctx, SB_ERR_INVALID, "rotary: null");
        if (p.heads < 1 || p.heads > 65535) return sb_fail(ctx, SB_ERR_INVALID, "rotary: 1 to 65535 heads");
        if (((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y)) & (size - 1)))
            return sb_fail(ctx, SB_ERR_SHAPE, "rotary: a base that is not aligned to its type");
        if (p.x == p.y && ((total > 1 && p.x_token_stride != p.y_token_stride) || (p.heads > 1 && p.x_head_stride != p.y_head_stride)))
            return sb_fail(ctx, SB_ERR_SHAPE, "rotary: in place with other strides");
        a.part[i] = {p.x, p.y, p.x_token_stride, p.x_head_stride, p.y_token_stride, p.y_head_stride, p.heads};
        a.heads += p.heads;
        bits |= reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y);
        if (total > 1) bits |= (uintptr_t)((p.x_token_stride | p.y_token_stride) * size);
        if (p.heads > 1) bits |= (uintptr_t)((p.x_head_stride | p.y_head_stride) * size);
    }
    bits |= (uintptr_t)(dim * size);
    if (!table->interleaved) bits |= (uintptr_t)(table->rotated / 2 * size);
    int n = 16 / size;
    while (n > 1 && (bits & (uintptr_t)(n * size - 1))) n /= 2;
    a.freq = table->freq; a.rotated = table->rotated; a.factor = table->factor; a.back = table->inverse;
    a.positions = positions; a.starts = starts; a.lens = lens; a.total = total;
    a.requests = requests; a.max_new = (int)max_new; a.dim = dim; a.st = ctx->dstate;
    a.slots = table->interleaved ? dim / (n > 1 ? n : 2) : (dim - table->rotated / 2) / n;
    a.by_slots = KvDiv(a.slots);
    a.by_heads = KvDiv(a.heads);
    // rows of a block: 16 blocks a multiprocessor, or as many rows as the table holds
    int64_t rows = total / (16 * ctx->sm_count);
    const int64_t most = RO_TABLE / (table->rotated / 2);
    if (rows > most) rows = most;
    if (rows < 1) rows = 1;
    if (rows > 64) rows = 64;
    a.rows = (int)rows;
    if (rows * a.heads * a.slots >= (1ll << 31)) return sb_fail(ctx, SB_ERR_SHAPE, "rotary: too many heads");
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    using B = __nv_bfloat16;
    if (f32 && table->interleaved) return n == 4 ? ro_launch<float, 4, true>(ctx, a) : n == 2 ? ro_launch<float, 2, true>(ctx, a) : ro_launch<float, 1, true>(ctx, a);
    if (f32) return n == 4 ? ro_launch<float, 4, false>(ctx, a) : n == 2 ? ro_launch<float, 2, false>(ctx, a) : ro_launch<float, 1, false>(ctx, a);
    if (table->interleaved)
        return n == 8 ? ro_launch<B, 8, true>(ctx, a) : n == 4 ? ro_launch<B, 4, true>(ctx, a) : n == 2 ? ro_launch<B, 2, true>(ctx, a) : ro_launch<B, 1, true>(ctx, a);
    return n == 8 ? ro_launch<B, 8, false>(ctx, a) : n == 4 ? ro_launch<B, 4, false>(ctx, a) : n == 2 ? ro_launch<B, 2, false>(ctx, a) : ro_launch<B, 1, false>(ctx, a);
}
