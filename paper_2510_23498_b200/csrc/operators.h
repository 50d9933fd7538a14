// Internal interface of the operators that work without a context: the gated linear recurrence (recurrence.cu), the residual step with its
// norms (residual.cu) and dropout (dropout.cu).  Their C entry points check the arguments and launch; nothing else of the library calls them.
#pragma once
#include <utility>

#include "common.cuh"

namespace mpode {

// records the message that mpode_operator_error returns (per host thread) and passes the status through
mpode_status operator_fail(mpode_status s, const char* format, ...);
// after a launch: the runtime's refusal as a status
mpode_status operator_launched(cudaError_t e, const char* entry);

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
inline bool known_dtype(mpode_dtype t) { return t == MPODE_F32 || t == MPODE_BF16 || t == MPODE_F16; }

// calls f with a value of the format's element type
template <typename F> inline cudaError_t with_low(mpode_dtype dt, F&& f) {
    if (dt == MPODE_F32) return f(float{});
    if (dt == MPODE_BF16) return f(__nv_bfloat16{});
    return f(__half{});
}

// A launch with its own status.  (Behind <<<>>> only the thread's last error could be asked, which an earlier call may have left.)
template <typename... P, typename... A> inline cudaError_t launch_grid(void (*kernel)(P...), unsigned grid, unsigned block, cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

// How many clusters of `blocks` blocks of this kernel the current device holds at once (-1 when that cannot be told).  Clusters beyond that number would run
// behind the others: the groups of SMs that a cluster has to fit into leave some of them idle.
inline int clusters_at_once(const void* kernel, dim3 block, size_t smem, int blocks) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)blocks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess &&
        (blocks <= 8 || cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) &&
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess)
        return n;
    (void)cudaGetLastError();
    return -1;
}

}  // namespace mpode
