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
    unsigned group_inverse;      // ceil(2^32 / group), for group > 1
    int row_tiles, splits;       // of the grid
    int chunk;                   // keys per CTA
    float scale_log2;            // softmax scale * log2(e)
    int window;
    float* part;                 // [tile][splits][rows][dim] unnormalised sums
    float2* part_ml;             // [tile][splits][rows] (running maximum, sum)
    unsigned* done;              // per tile: chunks finished
    SbDeviceState* st;
};


// kv8_prompt.cu: rows of one cache head on the tensor cores of the fifth generation, dim <= 128
sb_status kv8_prompt(sb_ctx* ctx, AtArgs a, int type, int64_t max_new, int64_t max_len);

#ifdef __CUDACC__
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
// power of two by which a bf16 query row with largest element (as bits) amax is scaled into fp16
__device__ __forceinline__ float at_query_scale(uint32_t amax) {
    const int ex = max(14, min(254, (int)(amax >> 7)));              // largest element in 2^(ex - 127) [1, 2)
    return __uint_as_float((uint32_t)min(254, 267 - ex) << 23);
}
// running power of two that is not below a value scale; 2^-e of such a 2^e
__device__ __forceinline__ float at_value_ref(float vmax) {
    return __uint_as_float(max((__float_as_uint(vmax) + 0x7fffffu) & 0x7f800000u, 0x00800000u));
}
__device__ __forceinline__ float at_value_inv(float vref) {
    return vref > 0.f ? __uint_as_float(0x7f000000u - __float_as_uint(vref)) : 0.f;
}
// the natural log of a row's sum; what its sums are multiplied with
__device__ __forceinline__ float at_lse(float m, float sum) {
    return sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
}
__device__ __forceinline__ float at_norm(float sum) {
    return sum > 0.f ? __fdiv_rn(1.f, sum) : (sum == 0.f ? 0.f : sum);
}
#endif
