// Rotary positions: pairs of a head's elements turned by an angle that grows with the position.
//
// A block takes a few rows (tokens) and finds their positions; a warp computes cos and sin of a row's angles once and turns its heads,
// of all parts (queries and keys), with them, or a share of its heads where rows are few. A lane keeps its place in a head,
// up to 16 bytes of each half ("half") or 16 bytes of neighbouring pairs, with cos and sin in registers, and goes over heads, a few of
// them side by side. One read and one write an element. An angle is position times frequency in
// 64 bits, with the products' rounding errors by fma: exact to fp32 for every 32-bit position. The bytes bound large calls, the
// chain of dependent reads small ones, so the first heads are fetched before the positions are known. Measured, bf16, 32 query and 8
// key heads of 128: 6 requests of up to 2048 tokens 41 us, 5.2 TB/s (a plain copy of as much: 33); 64 single tokens 4.2 us, where a form
// whose blocks shared one row's angles took 3.3 (and 18 in the next case, 40 in the first). 8 of up to 700 tokens, 16 + 16 heads of 80, neighbouring pairs backwards, 12 us, where the blocks of one round still start and end apart.
#include "kv8.cuh"
#include "launch.cuh"

namespace {

constexpr int RO_THREADS = 256;
constexpr int RO_WARPS = RO_THREADS / 32;
constexpr int RO_ROWS = 32;                  // of a block at most

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
    int groups;                              // of a row's heads, a warp each: 1, 2, 4 or 8
    int slots;                               // of a head: pieces that one thread takes
    float factor;
    int back;
    SbDeviceState* st;
};

// cos and sin of p * f: in turns, p f / 2 pi with both products' rounding errors and 1 / 2 pi as a sum of two, less whole ones
__device__ __forceinline__ float2 ro_turn(int p, float f, float factor, bool back) {
    const double x = (double)p, y = (double)f;
    const double g = y * 0.15915494309189535, t = x * g;
    const double rest = fma(x, fma(y, 0.15915494309189535, -g) + y * -9.839338337591243e-18, fma(x, g, -t));
    float s, c;
    sincospif(2.f * (float)((t - rint(t)) + rest), &s, &c);
    return make_float2(c * factor, (back ? -s : s) * factor);
}

__device__ __forceinline__ float ro_float(float x) { return x; }
__device__ __forceinline__ float ro_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T ro_round(float x);
template <> __device__ __forceinline__ float ro_round<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 ro_round<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
// N elements of one access, as 32-bit words (N = 1: the element)
template <typename T, int N>
struct RoVec {
    static constexpr int W = N * (int)sizeof(T) / 4;
    uint32_t w[W];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (W == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(p);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        } else if constexpr (W == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            w[0] = x.x; w[1] = x.y;
        } else w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
    // elements 2 i and 2 i + 1 as fp32, and back with one rounding
    __device__ __forceinline__ void two(int i, float& lo, float& hi) const {
        if constexpr (sizeof(T) == 2) {
            lo = bf16lo(w[i]);
            hi = bf16hi(w[i]);
        } else {
            lo = __uint_as_float(w[2 * i % W]);
            hi = __uint_as_float(w[(2 * i + 1) % W]);
        }
    }
    __device__ __forceinline__ void put(int i, f32x2 x) {
        float lo, hi;
        upk2(x, lo, hi);
        if constexpr (sizeof(T) == 2) w[i] = u32(__floats2bfloat162_rn(lo, hi));
        else {
            w[2 * i % W] = __float_as_uint(lo);
            w[(2 * i + 1) % W] = __float_as_uint(hi);
        }
    }
};
template <typename T>
struct RoVec<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = v; }
};

// N: elements of an access. INTER: neighbouring pairs, N / 2 of them an access.
template <typename T, int N, bool INTER>
__global__ void __launch_bounds__(RO_THREADS, 4)
rotary_kernel(const RoArgs a) {
    extern __shared__ __align__(16) unsigned char ro_smem[];
    sb_let_next();
    sb_after_previous();
    const int half = a.rotated / 2;
    __shared__ int pos[2 * RO_ROWS];                                 // [rows], and whether there is one
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = (int)min((int64_t)a.rows, a.total - row0);
    const int tid = threadIdx.x;
    using V = RoVec<T, N>;
    constexpr int WIDE = INTER && N == 1 ? 2 : N;                    // elements of a slot's first access (N = 1: a pair one by one)
    constexpr int NC = INTER ? WIDE / 2 : N;                         // angles of a slot
    constexpr int BATCH = 2;                                         // heads side by side
    const int warp = tid >> 5, lane = tid & 31, group = warp % a.groups;
    float2* table = reinterpret_cast<float2*>(ro_smem) + warp * half;        // this warp's
    const int across = a.slots <= 32 ? 32 / a.slots : 1, lane_head = a.slots <= 32 ? lane / a.slots : 0;
    const int slot0 = a.slots <= 32 ? lane - lane_head * a.slots : lane, step = across * a.groups;
    const bool works = lane_head < across && slot0 < a.slots;
    auto is_turned = [&](int slot) { return INTER ? WIDE * slot < a.rotated : N * slot < half; };
    auto place = [&](int slot) { return INTER ? WIDE * slot : is_turned(slot) ? N * slot : a.rotated + N * slot - half; };
    auto partner = [&](int slot) { return INTER ? WIDE - N : is_turned(slot) ? half : 0; };       // from a piece to its partner
    auto load = [&](int k, int r, int slot, int h0, V (&v)[BATCH], V (&w)[BATCH]) {
        const RoPart& part = a.part[k];
        const T* x = static_cast<const T*>(part.x) + (row0 + r) * part.xt + place(slot);
        const int apart = partner(slot);
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (h0 + b * step < part.heads) {
                const T* from = x + (int64_t)(h0 + b * step) * part.xh;
                v[b].load(from);
                if (apart) w[b].load(from + apart);
            }
    };
    // this warp's first heads, before their position is known
    V v[BATCH], w[BATCH];
    const int h_first = group * across + lane_head, r_first = warp / a.groups;
    if (works && r_first < rows) load(0, r_first, slot0, h_first, v, w);
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
            const int len = a.lens[b];
            if (s >= row0 + rows || s + n <= row0 || !fits(s, n, len)) continue;
            for (int64_t i = max(s, row0); i < min(s + n, row0 + rows); ++i) {
                pos[i - row0] = (int)(len - n + (i - s));
                pos[a.rows + (i - row0)] = 1;
            }
        }
    }
    __syncthreads();
    for (int r = r_first; r < rows; r += RO_WARPS / a.groups) {
        if (!pos[a.rows + r]) continue;
        const int p = pos[r];
        __syncwarp();
        for (int i = lane; i < half; i += 32) table[i] = ro_turn(p, a.freq[i], a.factor, a.back);
        __syncwarp();
        if (!works) continue;
        for (int slot = slot0; slot < a.slots; slot += 32) {
            const bool turned = is_turned(slot);
            const int d = place(slot), apart = partner(slot);
            // Packed for two elements at once. "half": cos, sin and -sin of angles 2 i, 2 i + 1; INTER: of angle i, (cos, cos) and (-sin, sin).
            constexpr int NK = N > 1 ? (INTER ? NC : NC / 2) : 1;
            f32x2 c2[NK], s2[NK], n2[INTER ? 1 : NK];
            float2 one = make_float2(1.f, 0.f);                      // N = 1: the angle
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                if (INTER || N == 1) {
                    const int at = N > 1 ? NC * slot + i : slot;
                    one = at < half ? table[at] : make_float2(1.f, 0.f);
                    c2[i] = pk2(one.x, one.x);
                    s2[i] = pk2(-one.y, one.y);
                } else {
                    const float4 t = turned ? *reinterpret_cast<const float4*>(table + N * slot + 2 * i) : make_float4(1.f, 0.f, 1.f, 0.f);
                    c2[i] = pk2(t.x, t.z);
                    s2[i] = pk2(t.y, t.w);
                    n2[i] = pk2(-t.y, -t.w);
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const RoPart& part = a.part[k];
                const T* x = static_cast<const T*>(part.x) + (row0 + r) * part.xt + d;
                T* y = static_cast<T*>(part.y) + (row0 + r) * part.yt + d;
                if (!turned && x == y) continue;
                for (int h0 = h_first; h0 < part.heads; h0 += BATCH * step) {
                    if (k > 0 || h0 > h_first || slot > slot0 || r > r_first) load(k, r, slot, h0, v, w);
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) {
                        if (h0 + b * step >= part.heads) continue;
                        T* to = y + (int64_t)(h0 + b * step) * part.yh;
                        if constexpr (N == 1) {
                            if (turned) {
                                const float uu = ro_float(v[b].v), ww = ro_float(w[b].v);
                                v[b].v = ro_round<T>(uu * one.x - ww * one.y);
                                w[b].v = ro_round<T>(ww * one.x + uu * one.y);
                            }
                        } else if constexpr (INTER) {
                            // a pair behind the rotated part is only copied: no product may touch what is not finite there
#pragma unroll
                            for (int i = 0; i < NK; ++i)
                                if (d + 2 * i < a.rotated) {
                                    float uu, ww;
                                    v[b].two(i, uu, ww);
                                    v[b].put(i, fma2(pk2(uu, ww), c2[i], mul2(pk2(ww, uu), s2[i])));
                                }
                        } else if (turned) {
#pragma unroll
                            for (int i = 0; i < NK; ++i) {
                                float p[2], q[2];
                                v[b].two(i, p[0], p[1]);
                                w[b].two(i, q[0], q[1]);
                                const f32x2 uu = pk2(p[0], p[1]), ww = pk2(q[0], q[1]);
                                v[b].put(i, fma2(uu, c2[i], mul2(ww, n2[i])));
                                w[b].put(i, fma2(ww, c2[i], mul2(uu, s2[i])));
                            }
                        }
                        v[b].store(to);
                        if (apart) w[b].store(to + apart);
                    }
                }
            }
            if (a.slots <= 32) break;
        }
    }
}

template <typename T, int N, bool INTER>
sb_status ro_launch(sb_ctx* ctx, const RoArgs& a) {
    const size_t smem = (size_t)RO_WARPS * (a.rotated / 2) * 8;
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
        if ((total > 1 && p.y_token_stride == 0) || (p.heads > 1 && p.y_head_stride == 0))
            return sb_fail(ctx, SB_ERR_SHAPE, "rotary: an output whose rows lie on one another");
        if (i == 1 && (p.y == parts[0].y || p.y == parts[0].x || p.x == parts[0].y))
            return sb_fail(ctx, SB_ERR_INVALID, "rotary: the output of one part is the other part");
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
    // warps: 16 a multiprocessor, from shares of a row's heads where rows are few; then rows of a warp up to four
    const int64_t warps = 16 * (int64_t)ctx->sm_count;
    for (a.groups = 1; a.groups < RO_WARPS && total * a.groups < warps && a.groups * 2 <= a.heads;) a.groups *= 2;
    int64_t rows = RO_WARPS / a.groups, each = total * a.groups / (4 * warps);
    rows *= each < 1 ? 1 : each > 4 ? 4 : each;
    a.rows = (int)(rows > RO_ROWS ? RO_ROWS : rows);
    SB_CUDA(ctx, cudaSetDevice(ctx->device));
    using B = __nv_bfloat16;
    if (f32 && table->interleaved) return n == 4 ? ro_launch<float, 4, true>(ctx, a) : n == 2 ? ro_launch<float, 2, true>(ctx, a) : ro_launch<float, 1, true>(ctx, a);
    if (f32) return n == 4 ? ro_launch<float, 4, false>(ctx, a) : n == 2 ? ro_launch<float, 2, false>(ctx, a) : ro_launch<float, 1, false>(ctx, a);
    if (table->interleaved)
        return n == 8 ? ro_launch<B, 8, true>(ctx, a) : n == 4 ? ro_launch<B, 4, true>(ctx, a) : n == 2 ? ro_launch<B, 2, true>(ctx, a) : ro_launch<B, 1, true>(ctx, a);
    return n == 8 ? ro_launch<B, 8, false>(ctx, a) : n == 4 ? ro_launch<B, 4, false>(ctx, a) : n == 2 ? ro_launch<B, 2, false>(ctx, a) : ro_launch<B, 1, false>(ctx, a);
}
