// mbarriers, bulk copies and tcgen05 instructions, shared by the kernels that use them.
#pragma once
#include <cuda.h>

#include "common.cuh"

typedef CUresult (*SbEncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Rows of row_elems elements, `pitch` bytes apart (a multiple of 16), as a map of boxes of box_elems x box_rows; what lies
// outside reads as zero.
inline sb_status t5_map(sb_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t rows,
                        int64_t row_elems, int64_t pitch, int box_elems, int box_rows, bool swizzle) {
    static SbEncodeTiledFn encode = nullptr;
    if (!encode) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        SB_CUDA(ctx, cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
        if (!fn || qres != cudaDriverEntryPointSuccess)
            return sb_fail(ctx, SB_ERR_CUDA, "the driver does not export cuTensorMapEncodeTiled");
        encode = reinterpret_cast<SbEncodeTiledFn>(fn);
    }
    const cuuint64_t dims[2] = {(cuuint64_t)row_elems, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)box_elems, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = encode(map, type, 2, const_cast<void*>(base), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return sb_fail(ctx, SB_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
    return SB_OK;
}
// rows of row_bytes bytes (a multiple of 16) in boxes of 128 bytes x box_rows with the 128-byte swizzle
inline sb_status t5_map_rows(sb_ctx* ctx, CUtensorMap* map, const void* base, int64_t rows, int64_t row_bytes, int box_rows) {
    return t5_map(ctx, map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, rows, row_bytes, row_bytes, 128, box_rows, true);
}

#ifdef __CUDACC__
constexpr unsigned long long T5_WAIT_NS = 2000ull * 1000 * 1000;      // a wait gives up after 2 s

__device__ __forceinline__ unsigned t5_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned long long t5_now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void t5_bar_init(unsigned bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void t5_bar_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void t5_bar_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool t5_bar_try(unsigned bar, unsigned parity) {
    unsigned ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool t5_bar_wait_slow(unsigned bar, unsigned parity, volatile int* abort_flag) {
    unsigned long long t0 = 0;
    for (unsigned spins = 0;; ++spins) {
        if (t5_bar_try(bar, parity)) return true;
        if (*abort_flag) return false;
        if ((spins & 63u) == 63u) {
            const unsigned long long now = t5_now_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > T5_WAIT_NS) { *abort_flag = 1; return false; }
        }
    }
}
// bounded wait: false (and the abort flag set) if the phase does not complete in time or another
// role has given up
__device__ __forceinline__ bool t5_bar_wait(unsigned bar, unsigned parity, volatile int* abort_flag) {
    if (t5_bar_try(bar, parity)) return true;
    return t5_bar_wait_slow(bar, parity, abort_flag);
}
// bounded wait for copies this thread has issued, whatever the other roles did: shared memory is
// not left while a copy may still land in it
__device__ __forceinline__ void t5_bar_drain(unsigned bar, unsigned parity) {
    const unsigned long long t0 = t5_now_ns();
    while (!t5_bar_try(bar, parity) && t5_now_ns() - t0 < T5_WAIT_NS) {}
}
// One lane of a converged warp. The warps that issue copies and products run their loops whole, with
// this predicate on the instructions alone: the operands then stay in uniform registers. In a
// branch of lane 0 the same thirteen instructions of a ring stage took 1066 cycles to issue.
__device__ __forceinline__ bool t5_elect() {
    unsigned p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void t5_load_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// contiguous bytes (a multiple of 16, both addresses 16-byte aligned)
__device__ __forceinline__ void t5_load_bulk(unsigned dst, const void* src, unsigned bytes, unsigned bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ unsigned t5_cta_rank() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned t5_cluster_size() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned t5_cluster_addr(unsigned own, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(own), "r"(rank));
    return r;
}
__device__ __forceinline__ void t5_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared-memory matrix descriptor of a K-major operand in the 128-byte swizzle: rows of 128 bytes,
// eight-row groups 1024 bytes apart. A step along K inside the 128 bytes adds its bytes to addr.
__device__ __forceinline__ unsigned long long t5_desc_sw128(unsigned addr) {
    return (unsigned long long)((addr >> 4) & 0x3fffu) | 1ull << 16 | (unsigned long long)(1024 >> 4) << 32 | 1ull << 46 |
           2ull << 61;
}
// 32 rows x 16 bytes without swizzle: eight-row groups 128 bytes apart
__device__ __forceinline__ unsigned long long t5_desc_rows16(unsigned addr) {
    return (unsigned long long)((addr >> 4) & 0x3fffu) | (unsigned long long)(128 >> 4) << 32 | 1ull << 46;
}
__device__ __forceinline__ void t5_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void t5_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 lanes x 32 columns of fp32 (the calling warp's quarter of the lanes)
__device__ __forceinline__ void t5_ld32(unsigned taddr, unsigned (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void t5_ld16(unsigned taddr, unsigned (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void t5_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
#endif
