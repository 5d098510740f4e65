// Launches in clusters, and launches that start while the kernel before them in the stream still runs.
#pragma once
#include "common.cuh"

// `early`: the kernel's blocks may become resident before the one ahead of it in the stream has ended, so they call sb_after_previous
// before they touch memory that another kernel writes, or writes that another reads, and do not read such memory by .nc or __ldg, which
// want it unchanged for as long as the kernel is there. A kernel that reads before its own wait what that one does not write (lora_up_kernel,
// kv8_prompt_sum_kernel) has to be let in by one that waits BEFORE it lets the next in (lora_down_kernel, kv8_prompt_kernel). cluster: blocks along x.
template <typename... P>
sb_status sb_launch(sb_ctx* ctx, void (*kernel)(P...), dim3 grid, unsigned threads, int smem, int cluster, bool early, P... args) {
    if (smem > 40 * 1024) SB_FUNC_ATTR(ctx, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (cluster > 8) SB_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchAttribute at[2];
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cfg.attrs = at;
    if (cluster > 1) {
        at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[cfg.numAttrs].val.clusterDim.x = cluster;
        at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    if (early) {
        at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
        ++cfg.numAttrs;
    }
    SB_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, args...));
    SB_LAUNCHED(ctx);
    return SB_OK;
}

#ifdef __CUDACC__
// Waits for the end of the kernel ahead in the stream. All blocks do, so that no later kernel passes either.
__device__ __forceinline__ void sb_after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets the next kernel's blocks become resident, if it was launched early, once all blocks of this one have called this or ended.
__device__ __forceinline__ void sb_let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
#endif
