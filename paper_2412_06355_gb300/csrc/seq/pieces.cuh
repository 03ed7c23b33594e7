// Elements of a tensor as float32 values: VEC of them in one load or store.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace dendsn {

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf16_low(uint32_t q) { return __uint_as_float(q << 16); }
__device__ __forceinline__ float bf16_high(uint32_t q) { return __uint_as_float(q & 0xffff0000u); }

// VEC elements as they lie in memory: 16 bytes where addresses allow it, else one element.
template <typename T, int VEC> struct Lot;
template <> struct Lot<float, 4> {
    float4 r;
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    __device__ __forceinline__ void set(const float (&v)[4]) { r = make_float4(v[0], v[1], v[2], v[3]); }
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <> struct Lot<float, 1> {
    float r;
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = r; }
    __device__ __forceinline__ void set(const float (&v)[1]) { r = v[0]; }
    __device__ __forceinline__ void zero() { r = 0.f; }
};
template <> struct Lot<__nv_bfloat16, 8> {
    uint4 r;
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(q[i]), v[2 * i + 1] = bf16_high(q[i]);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        r = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
    __device__ __forceinline__ void zero() { r = make_uint4(0u, 0u, 0u, 0u); }
};
template <> struct Lot<__nv_bfloat16, 1> {
    uint16_t r;
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __uint_as_float((uint32_t)r << 16); }
    __device__ __forceinline__ void set(const float (&v)[1]) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v[0]);
        r = *reinterpret_cast<const uint16_t *>(&h);
    }
    __device__ __forceinline__ void zero() { r = 0; }
};

// Two values as e4m3 codes, rounded to nearest even, at most 448 in size.
__device__ __forceinline__ uint16_t e4m3_pair(float lo, float hi) {
    uint16_t q;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(hi), "f"(lo));
    return q;
}

}  // namespace dendsn
