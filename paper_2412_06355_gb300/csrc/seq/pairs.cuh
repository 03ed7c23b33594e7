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
// The largest value of an e4m3 code is 448: 448 / top and top / 448 as divisions round them, for top from 2^-110 on.
// Approximate quotients corrected by what they leave (Markstein's division step). A division each, of which every
// lane of a warp has two for its 8 elements, cost the optimizer's step with 8-bit states 5%.
__device__ __forceinline__ float from_top(float top) {
    const float t = top * 0x1p-9f, r = rcp_fast(t), q = r * 0.875f;      // (1 / top itself would leave float32's normal numbers)
    return fmaf(fmaf(-q, t, 0.875f), r, q);
}
__device__ __forceinline__ float to_top(float top) {
    const float q = top * (1.f / 448.f);
    return fmaf(fmaf(-q, 448.f, top), 1.f / 448.f, q);
}
// Roots from the hardware's reciprocal root (of denormal numbers too) and one step of Newton's: the square root's own
// bits for every number from 2^-102 on; below that what the step corrects by is a denormal number itself, and the root
// within some 2^-20. The root of zero is zero.
__device__ __forceinline__ float rsqrt_fast(float v) {
    float r;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(fmaxf(v, 0x1p-149f)));
    return r;
}
__device__ __forceinline__ F2 root_of(F2 v) {
    const F2 y(rsqrt_fast(v.x()), rsqrt_fast(v.y())), near = mul(v, y);
    return fma(fma(mul(near, both(-1.f)), near, v), mul(y, both(0.5f)), near);
}
// The larger of three (of NaN and a number, the number).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

}  // namespace dendsn
