// What a warp goes on with after a wait that ran out for some of its lanes, or for all. Built and called by
// tests/test_gpu_delta_waits.py. Every wait here comes true or ends by its own limit, and the kernels return.
#include <cuda_runtime.h>

#include "seq/tc_one.cuh"

using namespace dendsn;

// Lanes that disagree, as where the clock cuts a wait off between two of them (which = 1), a wait that comes true
// (0), and one at which nothing arrives (2). out[lane]: what the lane goes on with; out[32]: lanes that issue.
__global__ void split_warp(int *out, int which) {
    __shared__ uint64_t bar;
    const uint32_t at = tc::smem_addr(&bar);
    if (threadIdx.x == 0) {
        tc::bar_init(at, 1);
        tc::bar_init_fence();
        if (which != 2) tc::bar_arrive(at);
    }
    __syncwarp();
    const bool ok = tc::warp_wait(which != 1 || threadIdx.x % 3 != 1, at, 0);
    out[threadIdx.x] = ok;
    if (ok && tc::elected()) atomicAdd(out + 32, 1);
}

extern "C" int run_split_warp(int *out, int which) {
    split_warp<<<1, 32>>>(out, which);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
