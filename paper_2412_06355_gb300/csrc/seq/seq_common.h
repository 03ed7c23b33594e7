// Shared by the token-sequence operators: status reporting of the C ABI, argument blocks,
// launcher declarations.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dendsn.h"

namespace dendsn {

// The calling thread's error message and the launch counter live in dendsn_capi.cu.
dendsn_status seq_fail(dendsn_status st, const char *fmt, ...);
void seq_count_launches(int n);

inline bool seq_aligned(const void *p, size_t a) {
    return (reinterpret_cast<uintptr_t>(p) % a) == 0;
}

#ifdef __CUDACC__
// Kernels launched by seq_launch overlap their launch with the end of the kernel before them in
// the stream: they call pdl_begin first, which lets the next one come up likewise and then waits
// for everything before (each kernel waits for its predecessor, so also for those before that).
__device__ __forceinline__ void pdl_begin() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t seq_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, int cluster, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
#endif

}  // namespace dendsn
