// Copies of a paged cache's tiles to shared memory, and the launch of the kernels that use them.
#ifndef UBP_ATTENTION_COPY_CUH_
#define UBP_ATTENTION_COPY_CUH_

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "ubp_attention.h"
#include "ubp_tc_common.cuh"

namespace ubp {

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *tm, int c0, int c1, int c2, int c3, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}

// Bounded wait of a whole warp: false if it ran out (two seconds of cycles: a warp may wait for as long as an item takes) or another
// one of the block had. The hardware suspends the warp for up to the hinted millisecond: without the hint it comes back after a
// microsecond or so, and twenty warps that ask again and again took the issue slots of those at work; a look at the global timer on
// the way cost thousands of cycles.
__device__ __forceinline__ bool attn_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, long long limit = 4000000000ll)
{
    long long t0 = 0;
    for (bool again = false;; again = true) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
        if (__all_sync(0xffffffffu, done)) return true;
        if (!again) t0 = clock64();
        else if (*abort_flag || clock64() - t0 > limit) break;
    }
    *abort_flag = 1;
    return false;
}

// Page of the box of `box` keys from j on, which lie in one page: out of the cache's range (its copy brings zeros) where no row of
// the item sees a key of it, or where the table names none.
__device__ __forceinline__ int attn_box_page(const AttnArgs &a, const AttnTiles &t, int b, int j, int box)
{
    if (j >= t.end || j + box <= a.kv0 || (j + box <= t.w0 && j >= a.sinks)) return a.pages;
    const int p = a.table[(a.common || j + box <= a.shared ? 0 : (int64_t)b * a.ldt) + (j >> a.pshift)];
    return (uint32_t)p < (uint32_t)a.pages ? p : a.pages;
}

// Tensor map of the keys or values (head values, tokens of a page, heads, pages), boxes of 64 values x `keys` tokens (a page's if
// it has fewer), 128-byte swizzle.
int attn_encode_cache(CUtensorMap *tm, const AttnArgs &a, const void *base, int dtype, int keys);

// A launch that may begin before the kernel in front of it has ended; dynamic shared memory is allowed once a device and kernel.
// cluster: blocks of a cluster (1: none).
template <typename K, typename... A>
int attn_launch(K kern, std::atomic<bool> (&done)[64], dim3 grid, int threads, size_t smem, int cluster, void *stream, const A &...args)
{
    cudaError_t e = cudaSuccess;
    if (smem > 48 * 1024) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
        if (dev < 0 || dev >= 64 || !done[dev]) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kern, args...);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) { set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}

}  // namespace ubp
#endif
