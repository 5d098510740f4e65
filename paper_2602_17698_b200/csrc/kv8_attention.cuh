// Pieces shared by the attention kernels over the 8-bit cache (kv8_attention.cu: few query rows,
// kv8_prompt.cu: many).
#pragma once
#include "kv8.cuh"

struct AtArgs {
    Kv8Geom g;
    const uint8_t *k, *v;
    const uint16_t *k_scale, *v_scale;
    const __nv_bfloat16* q;
    int64_t q_token_stride, q_head_stride;
    __nv_bfloat16* o;
    int64_t o_token_stride, o_head_stride;
    float* lse;
    int group;                   // query heads per cache head
    KvDiv by_group;
    int row_tiles;               // of a request with max_new new tokens
    KvDiv by_row_tiles;
    float scale_log2;            // softmax scale * log2(e); kernels take its sign into the queries (at_query_scale)
    int window;
    float* part;                 // two slots per CTA: unnormalised sums of an item's piece
    float2* part_ml;             // and its rows' (reference, sum of weights)
    unsigned* done;              // per item: pieces finished
    int least;                   // units of a share at least
    SbDeviceState* st;
};


// kv8_prompt.cu: many rows of one cache head on the tensor cores of the fifth generation, dim <= 128
sb_status kv8_prompt(sb_ctx* ctx, AtArgs a, int type, int64_t max_new, int64_t max_len);

#ifdef __CUDACC__
// ---- who does what -------------------------------------------------------------------------------
// An item is a tile of query rows (new tokens x query heads of one cache head) of a request and a
// cache head; its work, in units, is its key steps and EXTRA for its queries and results. The units of
// all items, one after the other (requests, row tiles, heads), are cut into equal shares, one per CTA:
// the requests' lengths are known on the device only, and a share costs the same whatever they are. An
// item that a share's border cuts leaves a piece per share in scratch, to be added in their order.
struct AtItem {
    Kv8Request rq;
    int b, r0, nrow;             // rows of the request's n * group from r0
    int lo, hi;                  // keys that some row sees, lo at the start of a scale block
    int steps;                   // 0: nothing to do
};
template <int ROWS, int KEYS>
__device__ __forceinline__ AtItem at_item(const AtArgs& a, int row_tile) {
    AtItem it;
    it.b = a.by_row_tiles.quot(row_tile);
    it.r0 = (row_tile - it.b * a.row_tiles) * ROWS;
    it.steps = 0;
    if (!kv8_request(a.g, it.b, it.rq, a.st)) return it;
    const int rows = it.rq.n * a.group;
    if (it.r0 >= rows) return it;
    it.nrow = min(ROWS, rows - it.r0);
    const int i1 = a.by_group.quot(it.r0 + it.nrow - 1);
    it.hi = it.rq.past + i1 + 1;
    it.lo = a.window > 0 ? max(0, it.rq.past + a.by_group.quot(it.r0) - a.window + 1) & ~(SB_KV8_BLOCK - 1) : 0;
    it.steps = (it.hi - it.lo + KEYS - 1) / KEYS;
    return it;
}
// quotients of the plan: 64 bits only where it takes them
__device__ __forceinline__ long long at_div(long long x, long long d) {
    return ((x | d) >> 32) == 0 ? (long long)((unsigned)x / (unsigned)d) : x / d;
}
// A share as its pieces of items; every warp walks through them by itself.
template <int ROWS, int KEYS, int EXTRA>
struct AtWalk {
    int row_tile, head, unit;                                        // where the piece starts
    int step0, count;                                                // its key steps: step0 .. + count of it.steps
    long long left, from;                                            // units left; the item's first unit of all
    bool first;                                                      // the share starts with this piece
    AtItem it;
    __device__ __forceinline__ int units() const { return it.steps ? it.steps + EXTRA : 0; }
    // the piece from `unit` on; its key steps may be none (only what an item costs besides)
    __device__ __forceinline__ void cut() {
        const int n = (int)min((long long)(units() - unit), left);
        step0 = max(0, unit - EXTRA);
        count = max(0, unit + n - EXTRA) - step0;
        left -= n;
    }
    __device__ __forceinline__ bool step(const AtArgs& a) {
        while (count == 0) {
            if (left <= 0) return false;
            first = false;
            unit = 0;
            from += units();
            if (++head >= a.g.heads || it.steps == 0) {
                head = 0;
                if (++row_tile >= a.row_tiles * a.g.requests) return false;
                it = at_item<ROWS, KEYS>(a, row_tile);
            }
            if (it.steps) cut();
        }
        return true;
    }
    __device__ __forceinline__ bool begin(const AtArgs& a, int row_tile_, int head_, int unit_, long long at, long long units_) {
        row_tile = row_tile_; head = head_; unit = unit_;
        from = at - unit;
        left = units_;
        first = true;
        it = at_item<ROWS, KEYS>(a, row_tile);
        count = 0;
        if (it.steps) cut();
        return step(a);
    }
    __device__ __forceinline__ bool next(const AtArgs& a) {
        count = 0;
        return step(a);
    }
};
__device__ __forceinline__ uint4 at_lds128(unsigned a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 at_lds64(unsigned a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
// Of a kernel that was launched before the one ahead of it in the stream has ended: waits for that
// end (all blocks do, so that no later kernel passes either); lets the next such kernel be launched.
__device__ __forceinline__ void at_after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void at_let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ float at_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t at_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Operand words hold e4m3 codes as they are, int8 codes with the sign bits flipped (at_flip).
template <int TYPE> __device__ __forceinline__ uint32_t at_flip(uint32_t w) { return TYPE == SB_KV_INT8 ? w ^ 0x80808080u : w; }
// bytes (0, 1) or (2, 3) of a word as two fp16
template <int TYPE, int HALF>
__device__ __forceinline__ uint32_t at_pair(uint32_t w) {
    if (TYPE == SB_KV_INT8) {
        const uint32_t u = __byte_perm(w, 0x64646464u, HALF ? 0x4342 : 0x4140);
        const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&u), __float2half2_rn(1152.f));
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    return e4m3x2_to_f16x2(HALF ? w >> 16 : w);
}
// power of two by which a bf16 query row with largest element (as bits) amax is scaled into fp16. Queries are
// multiplied with at_signed of it, scores with |scale| over it: the factor of a block's scores is never negative, so
// the largest score of a block is the largest product's.
__device__ __forceinline__ float at_query_scale(uint32_t amax) {
    const int ex = max(14, min(254, (int)(amax >> 7)));              // largest element in 2^(ex - 127) [1, 2)
    return __uint_as_float((uint32_t)min(254, 267 - ex) << 23);
}
__device__ __forceinline__ float at_signed(float up, float scale_log2) { return copysignf(up, scale_log2); }
// ---- the weights of the second product ----
// A weight 2^(score - m) times its value scale times `inv`, a power of two per row, is what fp16 holds. A weight is at most
// 2^8 (AT_SLACK), so a row whose value scales stay below AT_TOP / inv needs no look at them. Where the reference
// m moves or that is passed, inv is chosen anew: by what the row's keys add, weight and scale together, so that a large
// scale under a small weight does not push the others out of fp16's range.
constexpr float AT_SLACK = 8.f;         // log2 of how far a row's maximum may run ahead of its reference
constexpr float AT_TOP = 128.f;
// 2^-e of a 2^e (0: none yet)
__device__ __forceinline__ float at_power_inv(float p) { return p > 0.f ? __uint_as_float(0x7f000000u - __float_as_uint(p)) : 0.f; }
// The new inv: `most` is the largest weight times value scale of the keys now, `held` 1 / inv of the keys so far (by the new
// reference). The largest becomes 8 to 16; vmax inv stays finite, and inv and its inverse normal numbers.
__device__ __forceinline__ float at_value_inv(float most, float held, float vmax) {
    const float top = fmaxf(fmaxf(most, held * 16.f), fmaxf(vmax * 0x1p-96f, 0x1p-115f));
    return __uint_as_float(0x7f000000u + (4u << 23) - ((__float_as_uint(top) + 0x7fffffu) & 0x7f800000u));
}
// the natural log of a row's sum; what its sums are multiplied with
__device__ __forceinline__ float at_lse(float m, float sum) {
    return sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
}
__device__ __forceinline__ float at_norm(float sum) {
    return sum > 0.f ? __fdiv_rn(1.f, sum) : (sum == 0.f ? 0.f : sum);
}
#endif
