// Arithmetic on pairs of float32 values, and the hardware's exponential and reciprocal.
#pragma once

#include <stdint.h>

namespace dendsn {

// Two float32 values in one 64-bit register, as the paired instructions take them.
struct F2 {
    uint64_t v;
    F2() = default;
    __device__ __forceinline__ explicit F2(uint64_t raw) : v(raw) {}
    __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ float x() const { return __uint_as_float((uint32_t)v); }
    __device__ __forceinline__ float y() const { return __uint_as_float((uint32_t)(v >> 32)); }
};
__device__ __forceinline__ F2 both(float v) { return F2(v, v); }
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
    F2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
    F2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
    F2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}
__device__ __forceinline__ float exp2_fast(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_fast(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// The larger of three (of NaN and a number, the number).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

}  // namespace dendsn
