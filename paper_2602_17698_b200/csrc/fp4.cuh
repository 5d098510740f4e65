// Layout of the microscaled 4-bit formats (host and device), and their conversions.
#pragma once
#include "common.cuh"

__host__ __device__ inline int fp4_block(int format) { return format == SB_FP4_MX ? 32 : 16; }
__host__ __device__ inline int64_t fp4_padded_cols(int64_t C) { return (C + 31) & ~int64_t(31); }
// scale tiles (128 rows x 4 blocks) along a row tile
__host__ __device__ inline int64_t fp4_scale_tiles(int64_t C, int format) {
    return (fp4_padded_cols(C) / fp4_block(format) + 3) / 4;
}

#ifdef __CUDACC__
// byte of the scale of (row r, block j); tiles: fp4_scale_tiles
__device__ __forceinline__ int64_t fp4_scale_at(int64_t r, int64_t j, int64_t tiles) {
    return ((r >> 7) * tiles + (j >> 2)) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (j & 3);
}
// eight values to eight codes, the first in the lowest four bits
__device__ __forceinline__ uint32_t fp4_pack8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// eight codes to four pairs of fp16 (exact)
__device__ __forceinline__ void fp4_unpack8(uint32_t codes, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}
// e4m3 of a non-negative number, at most 448; and back
__device__ __forceinline__ uint32_t e4m3_of(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
    return r & 0xffu;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
    float f;
    asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"((uint16_t)(h & 0xffffu)));
    return f;
}
// the power of two an e8m0 byte stands for (255: NaN)
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
    return byte == 255 ? __uint_as_float(0x7fffffffu) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}
#endif
