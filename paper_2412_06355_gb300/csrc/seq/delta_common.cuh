// What the kernels of the gated delta rule share: arguments, where sequences and chunks lie, single values.
#pragma once

#include <cuda_bf16.h>

#include "delta_plan.h"
#include "fragments.cuh"
#include "seq_common.h"

namespace dendsn {
namespace delta {

constexpr int C = kDeltaChunk;
constexpr float kLeastGate = -200.f;       // exp of it is 0 in float32

// Places in a chunk's gate values.
enum { kFirst = 0, kRest = 64, kBeta = 128, kHigh = 192, kLow = 256, kKeep = 320 };

struct Args {
    int32_t T, B, Hk, Hv, Dk, Dv, layout;
    float scale;
    const int32_t *offsets;
    DeltaPlan p;
};

struct Sequence {
    int64_t row, step;         // its first token, tokens between two of its own
    int64_t slot;              // its first chunk's
    int32_t length;
};

__device__ __forceinline__ Sequence sequence(const Args &a, int b) {
    Sequence s;
    if (a.layout == DENDSN_DELTA_PACKED) {
        const int32_t lo = min(max(a.offsets[b], 0), a.T), hi = min(max(a.offsets[b + 1], lo), a.T);
        s.row = lo, s.step = 1, s.length = hi - lo;
        s.slot = lo / C + b;
    } else {
        const bool time = a.layout == DENDSN_DELTA_TIME;
        s.row = time ? b : (int64_t)b * a.T, s.step = time ? a.B : 1, s.length = a.T;
        s.slot = (int64_t)b * ((a.T + C - 1) / C);
    }
    return s;
}

// Which sequence a chunk's slot belongs to; false: to none. A packed sequence from token lo on has the
// slots from lo / 64 + (its number) on: no two meet, and the last one's stay below T / 64 + B.
__device__ __forceinline__ bool locate(const Args &a, int64_t slot, int *b, int *chunk, Sequence *s) {
    if (a.layout == DENDSN_DELTA_PACKED) {
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (min(max(a.offsets[mid], 0), a.T) / C + mid <= slot) lo = mid;
            else hi = mid - 1;
        }
        *b = lo;
    } else {
        *b = (int)(slot / ((a.T + C - 1) / C));
    }
    *s = sequence(a, *b);
    const int64_t c = slot - s->slot;
    *chunk = (int)c;
    return c >= 0 && c * C < s->length;
}

template <typename T>
__device__ __forceinline__ float value(const T *p) { return __bfloat162float(*p); }
template <>
__device__ __forceinline__ float value<float>(const float *p) { return *p; }

template <typename T>
__device__ __forceinline__ void put(T *p, float v);
template <>
__device__ __forceinline__ void put<float>(float *p, float v) { *p = v; }
template <>
__device__ __forceinline__ void put<__nv_bfloat16>(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

constexpr int kWide = 2 * kCell;           // bytes of an 8 x 8 block of float32

}  // namespace delta

// The states (and their gradients) from chunk to chunk, for all sequences and heads: delta_walk.cu.
cudaError_t delta_walk_forward(const delta::Args &a, bool bf16, const void *v, const float *s0, void *o, float *last, uint8_t *kept, bool keep,
                               cudaStream_t s);
cudaError_t delta_walk_backward(const delta::Args &a, bool bf16, const void *go, const float *glast, const uint8_t *kept, uint8_t *scratch,
                                float *gs0, cudaStream_t s);

}  // namespace dendsn
