// Host-side pieces that every translation unit of the library launches its kernels with.
#ifndef FLASHBEV_LAUNCH_CUH_
#define FLASHBEV_LAUNCH_CUH_

#include <cuda_runtime.h>
#include <stdlib.h>

#include <atomic>

namespace flashbev_host {

// What flashbev_last_launch_count and flashbev_last_kernel_name report.
inline thread_local int t_last_launches = 0;
inline thread_local const char *t_last_kernel = "none";

// Number of SMs of the current device (cached per device; 148 on a B200).
inline int sm_count()
{
    static std::atomic<int> cached[64];  // 0: not asked yet (concurrent callers may both ask: same answer)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return 148;
    }
    int n = cached[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            n = 148;
        }
        cached[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

inline int use_pdl() { return getenv("FLASHBEV_NO_PDL") ? 0 : 1; }

// A kernel whose CTAs may be placed while the kernel before it in the stream drains; it waits for that one's end itself.
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid, cfg.blockDim = block, cfg.dynamicSmemBytes = smem, cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    if (use_pdl()) cfg.attrs = attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace flashbev_host

#endif  // FLASHBEV_LAUNCH_CUH_
