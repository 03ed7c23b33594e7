// Single operations of the optimizer's step, over all mantissas. Built and called by tests/test_gpu_adamw_codes.py.
#include <cuda_runtime.h>
#include <stdint.h>

#include "seq/pairs.cuh"

using namespace dendsn;

// Floats whose bits are from + i, i < count: how many of 448 / x, and of x / 448, differ from the division's.
__global__ void quotients(uint32_t from, uint32_t count, uint32_t *wrong) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= count) return;
    const float x = __uint_as_float(from + i);
    if (from_top(x) != __fdiv_rn(448.f, x)) atomicAdd(wrong, 1u);
    if (to_top(x) != __fdiv_rn(x, 448.f)) atomicAdd(wrong + 1, 1u);
}

// The same of roots: wrong[0] differ from the square root's, wrong[1] are further off than 2^-19 of it.
__global__ void roots(uint32_t from, uint32_t count, uint32_t *wrong) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= count) return;
    const float x = __uint_as_float(from + i), want = __fsqrt_rn(x), got = root_of(both(x)).x();
    if (got != want) atomicAdd(wrong, 1u);
    if (!(fabsf(got - want) <= want * 0x1p-19f)) atomicAdd(wrong + 1, 1u);
}

extern "C" int run_roots(uint32_t from, uint32_t count, uint32_t *wrong) {
    roots<<<(count + 255) / 256, 256>>>(from, count, wrong);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
extern "C" int run_quotients(uint32_t from, uint32_t count, uint32_t *wrong) {
    quotients<<<(count + 255) / 256, 256>>>(from, count, wrong);
    const cudaError_t e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
