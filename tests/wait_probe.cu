// Waits that run out, in kernels of their own: maps of the scan that a block of the cluster never
// sends, and a barrier at which nothing arrives. Built and called by tests/test_gpu_waits.py. Every
// wait here ends by its own limit, and the kernels return.
#include <cuda_runtime.h>

#include "seq/scan_fold.cuh"
#include "seq/tc.cuh"

using namespace dendsn;

// Two blocks, 16 segments of 16 pairs. Block 1 sends nothing. Block 0's buffers hold maps of
// another pass, which say that a sequence starts: h = 7.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(256) lost_maps(float2 *out, int passes, int silent) {
    __shared__ ScanShared<true> sh;
    const int rank = blockIdx.x, me = threadIdx.x / 16, cp = threadIdx.x % 16;
    for (int i = threadIdx.x; i < 2 * 8 * 32; i += 256) {
        (&sh.block[0][0][0])[i] = Map{both(1.f), both(7.f)};
        (&sh.block_flag[0][0][0])[i] = kCut;
    }
    __syncthreads();
    enter_cluster<true>(sh, 2, 16);
    if (rank != silent) {
        F2 carry = both(1.f);
        for (int pass = 0; pass < passes; ++pass) {
            bool cuts;
            // every segment doubles the state; a sequence starts in segment 12 of the last pass
            const bool cut = pass == passes - 1 && me == 12;
            const F2 in = fold<true, true, 16>(sh, 2, me, cp, 16, rank, pass, both(2.f), both(cut ? 5.f : 0.f), cut ? kCut : 0, carry, cuts);
            out[((rank * passes + pass) * 16 + me) * 16 + cp] = make_float2(in.x(), in.y());
        }
    }
    leave_cluster<true>(sh);
}

__global__ void no_arrival(int *result) {
    __shared__ uint64_t bar;
    tc::bar_init(tc::smem_addr(&bar), 1);
    tc::bar_init_fence();
    *result = tc::bar_wait(tc::smem_addr(&bar), 0) ? 1 : 2;
}

__global__ void landing(int *us) {
    const uint64_t began = now_ns();
    let_land();
    *us = (int)((now_ns() - began) / 1000);
}

extern "C" int run_landing(int *us) {
    landing<<<1, 1>>>(us);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
extern "C" int run_lost_maps(float *out, int passes, int silent) {
    lost_maps<<<2, 256>>>(reinterpret_cast<float2 *>(out), passes, silent);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
extern "C" int run_no_arrival(int *result) {
    no_arrival<<<1, 1>>>(result);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
