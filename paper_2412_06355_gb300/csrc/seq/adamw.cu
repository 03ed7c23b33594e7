// One step of AdamW over many tensors at once:
//   g' = g min(1, max_norm / |g|)           (|g| over all tensors; where clipping is on)
//   m += (1 - beta1) (g' - m),  v += (1 - beta2) (g'^2 - v),  t = step + 1
//   p = p (1 - lr decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
// with states in float32, or m and sqrt(v) as e4m3 codes with a float32 scale for each 256 elements
// (the largest becomes 448). A code is drawn from the two neighbours of its value so that the
// expectation of m and of v is right: a step moves a state by a thousandth, far less than the
// distance of two codes, and would be lost in rounding to the nearest. In the quotient sqrt(v) counts as at least
// the value of the smallest code, 2^-9 of the scale that was read.
//
// Bound by memory: every state is read and written once, in one launch for all tensors. Tensors are
// cut into chunks of 4096 elements; a table in device memory says which tensor a chunk belongs to, and
// the gradients' addresses, which change from step to step, come as the launch's arguments. A warp
// takes 256 elements at a time, 8 neighbours a lane, so that a scale's elements are one warp's.
// Clipping reads the gradients once more before (a launch that leaves one float64 sum a block).
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "pairs.cuh"
#include "pieces.cuh"
#include "seq_common.h"
#include "tc.cuh"

namespace dendsn {
namespace {

constexpr int kBlock = 256;            // elements of a warp's turn, and of a scale
constexpr int kChunk = 4096;           // elements of a place in the table
constexpr int kTurn = 2048;            // elements of a block's turn, half of that: what blocks are dealt
constexpr int kThreads = 256;
constexpr int kGrads = 500;            // tensors of a launch: their gradients' addresses are its arguments
constexpr int kMostBlocks = 152 * 4;   // sums of squares a step can have; blocks of the norm's launch
// Blocks of the update on an SM. Float32 states are bound by memory: 24 warps of 80 registers (16 of 128: 730 us
// against 660 at 2^27 elements). With states in 8 bits 16 warps of 128 registers with three pieces on their way are
// faster than 24 of 80 with two (2^29 elements: 1680 us against 1910).
constexpr int resident(bool eight) { return eight ? 2 : 3; }
constexpr uint32_t kStride = 0x9E3779B1u;

enum : int32_t { kParamBf16 = 1, kWide = 2 };

struct Tensor {
    void *param, *m, *v;
    float *scales;
    __nv_bfloat16 *copy;
    int64_t n;
    int32_t first;             // its first chunk
    int32_t flags;
    float decay;
    int32_t pad;
};
static_assert(sizeof(Tensor) == 64, "one tensor's entry");

// The device table: a header, the sums of squares of each block, the tensors, the tensor of each chunk.
struct Header {
    uint32_t ticket;           // blocks of a launch that have read the step; 0 between launches
    uint32_t pad[15];
};
constexpr size_t kSumsAt = sizeof(Header), kTensorsAt = kSumsAt + kMostBlocks * sizeof(double);

// Addresses of gradients, with 1 added where a gradient is bfloat16; 0: none, the tensor stays as it is.
struct Grads {
    uint64_t at[kGrads];
};

struct Step {
    uint8_t *plan;
    int64_t *step;
    const float *lr_at;        // or NULL: lr
    float *norm;               // or NULL
    int32_t tensors, first;    // of the plan; the first of this launch
    int32_t turn, turns;       // of this launch: the first, and the one behind the last
    int32_t sums;              // sums of squares in the table (0: no clipping)
    bool last;                 // launch of the step
    float lr, eps, max_norm, rest1, rest2;
    float log1_hi, log1_lo, log2_hi, log2_lo;     // logarithms of the betas
    uint32_t seed;
};

__device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x6A09E667u;
    return (h ^ (h >> 15)) * 0xADF85459u;
}
// ... with the upper half mixed into the lower.
__device__ __forceinline__ uint32_t mixed(uint32_t h) {
    h = mix(h);
    return h ^ (h >> 16);
}

// 8 elements of a lane: neighbours (WIDE), or every 32nd of the block's, as far as there are.
template <bool WIDE>
__device__ __forceinline__ int element(int lane, int j) { return WIDE ? lane * 8 + j : j * 32 + lane; }

template <bool WIDE>
__device__ __forceinline__ void load8(float (&v)[8], const float *p, int lane, int left) {
    if (WIDE) {
        uint32_t q[8] = {};
        if (lane * 8 < left) tc::load32(q, p + lane * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(q[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j * 32 + lane < left ? p[j * 32 + lane] : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void load8(float (&v)[8], const __nv_bfloat16 *p, int lane, int left) {
    if (WIDE) {
        Lot<__nv_bfloat16, 8> q;
        q.zero();
        if (lane * 8 < left) q = reinterpret_cast<const Lot<__nv_bfloat16, 8> *>(p)[lane];
        q.get(v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j * 32 + lane < left ? __bfloat162float(p[j * 32 + lane]) : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store8(const float (&v)[8], float *p, int lane, int left) {
    if (WIDE) {
        uint32_t q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = __float_as_uint(v[j]);
        if (lane * 8 < left) tc::store32(p + lane * 8, q);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < left) p[j * 32 + lane] = v[j];
    }
}
template <bool WIDE>
__device__ __forceinline__ void store8(const float (&v)[8], __nv_bfloat16 *p, int lane, int left) {
    if (WIDE) {
        Lot<__nv_bfloat16, 8> q;
        q.set(v);
        if (lane * 8 < left) reinterpret_cast<Lot<__nv_bfloat16, 8> *>(p)[lane] = q;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < left) p[j * 32 + lane] = __float2bfloat16_rn(v[j]);
    }
}
// Codes as they lie: two words of four.
template <bool WIDE>
__device__ __forceinline__ void load_codes(uint32_t (&q)[2], const uint8_t *p, int lane, int left) {
    q[0] = q[1] = 0;
    if (WIDE) {
        if (lane * 8 < left) {
            const uint2 r = reinterpret_cast<const uint2 *>(p)[lane];
            q[0] = r.x, q[1] = r.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < left) q[j >> 2] |= (uint32_t)p[j * 32 + lane] << (j & 3) * 8;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store_codes(const uint32_t (&q)[2], uint8_t *p, int lane, int left) {
    if (WIDE) {
        if (lane * 8 < left) reinterpret_cast<uint2 *>(p)[lane] = make_uint2(q[0], q[1]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 32 + lane < left) p[j * 32 + lane] = (uint8_t)(q[j >> 2] >> (j & 3) * 8);
    }
}
__device__ __forceinline__ void decode(float (&v)[8], const uint32_t (&q)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(q[i >> 1] >> (i & 1) * 16)));
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}

// A code is what a float's leading bits are when its value is brought down by 2^-120: e4m3's exponents then are
// float32's lowest, and the codes below 2^-6 its denormal numbers.
constexpr float kDown = 0x1p-120f, kUp = 0x1p120f;
// The low bytes of four words, and their high bytes.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t high_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
// The largest size of three, a NaN above them all.
__device__ __forceinline__ float top_of(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// The larger of two, a NaN above all.
__device__ __forceinline__ float at_least(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ uint32_t warp_top(uint32_t t) {
#pragma unroll
    for (int o = 16; o; o >>= 1) t = max(t, __shfl_xor_sync(0xffffffffu, t, o));
    return t;
}
struct Scalars {
    float factor, rate, inverse_root, lr;
    uint32_t start;
};

// 1 - beta^t; the product of t and the logarithm keeps the bits below a float's.
__device__ __forceinline__ float rest_of_power(float t, float hi, float lo) {
    const float a = t * hi;
    return -expm1f(a + (fmaf(t, hi, -a) + t * lo));
}

// A lane's share of 256 elements.
template <bool EIGHT>
struct Share {
    float g[8], p[8];
    float m[EIGHT ? 1 : 8], v[EIGHT ? 1 : 8];
    uint32_t qm[2], qv[2];
    float2 scale;
    int left;
};

template <bool EIGHT, bool WIDE>
__device__ __forceinline__ void load(Share<EIGHT> &r, const Tensor &x, uint64_t grad, int64_t at, int lane) {
    const int left = r.left = (int)min((int64_t)kBlock, x.n - at);
    if (grad & 1) load8<WIDE>(r.g, reinterpret_cast<const __nv_bfloat16 *>(grad - 1) + at, lane, left);
    else load8<WIDE>(r.g, reinterpret_cast<const float *>(grad) + at, lane, left);
    if (x.flags & kParamBf16) load8<WIDE>(r.p, static_cast<const __nv_bfloat16 *>(x.param) + at, lane, left);
    else load8<WIDE>(r.p, static_cast<const float *>(x.param) + at, lane, left);
    if constexpr (EIGHT) {
        load_codes<WIDE>(r.qm, static_cast<const uint8_t *>(x.m) + at, lane, left);
        load_codes<WIDE>(r.qv, static_cast<const uint8_t *>(x.v) + at, lane, left);
        r.scale = *reinterpret_cast<const float2 *>(x.scales + at / kBlock * 2);
    } else {
        load8<WIDE>(r.m, static_cast<const float *>(x.m) + at, lane, left);
        load8<WIDE>(r.v, static_cast<const float *>(x.v) + at, lane, left);
    }
}

template <bool WIDE>
__device__ __forceinline__ void update(Share<false> &r, const Tensor &x, int64_t at, int lane, const Scalars &c, const Step &s, uint32_t) {
    const int left = r.left;
    const float kept = fmaf(-c.lr, x.decay, 1.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float g = r.g[j] * c.factor;
        r.m[j] = fmaf(s.rest1, g - r.m[j], r.m[j]);
        r.v[j] = fmaf(s.rest2, fmaf(g, g, -r.v[j]), r.v[j]);
        r.p[j] = fmaf(r.p[j], kept, -__fdiv_rn(c.rate * r.m[j], fmaf(sqrtf(r.v[j]), c.inverse_root, s.eps)));
    }
    if (x.flags & kParamBf16) store8<WIDE>(r.p, static_cast<__nv_bfloat16 *>(x.param) + at, lane, left);
    else store8<WIDE>(r.p, static_cast<float *>(x.param) + at, lane, left);
    if (x.copy) store8<WIDE>(r.p, x.copy + at, lane, left);
    store8<WIDE>(r.m, static_cast<float *>(x.m) + at, lane, left);
    store8<WIDE>(r.v, static_cast<float *>(x.v) + at, lane, left);
}
// With states in 8 bits it is instructions that bound the step, so they work on pairs. m, v and the root are within an
// ulp or two of the formulas' operations rounded one by one (the assembler joins products with sums), which decides one
// code in a million. (2^29 elements: 1685 us; one by one and with each code's exponent looked at, 100 instructions an
// element, 2090.)
template <bool WIDE>
__device__ __forceinline__ void update(Share<true> &r, const Tensor &x, int64_t at, int lane, const Scalars &c, const Step &s, uint32_t start) {
    const int left = r.left;
    const F2 kept = both(fmaf(-c.lr, x.decay, 1.f)), rate = both(-c.rate), inverse_root = both(c.inverse_root), eps = both(s.eps);
    // What v's smallest code stands for: a v whose code was drawn as zero may be as large, and m's code beside it is not
    // zero. (Gradients of 2^-20 of the block's largest, 400 steps: one of 751 lr without this, 3.5 with it.)
    const float least = r.scale.y * 0x1p-9f;
    const F2 scale_m = both(r.scale.x), scale_v = both(r.scale.y), factor = both(c.factor), rest1 = both(s.rest1), rest2 = both(s.rest2), minus = both(-1.f);
    float mc[8], vc[8];
    decode(mc, r.qm);
    decode(vc, r.qv);
    F2 m[4], root[4];
    float top_m = 0.f, top_v = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const F2 g = mul(F2(r.g[2 * j], r.g[2 * j + 1]), factor), old = mul(F2(mc[2 * j], mc[2 * j + 1]), scale_m);
        m[j] = add(mul(fma(old, minus, g), rest1), old);
        const F2 w = mul(F2(vc[2 * j], vc[2 * j + 1]), scale_v), w2 = mul(w, w);
        const F2 v = add(mul(fma(w2, minus, mul(g, g)), rest2), w2);
        root[j] = root_of(v);
        const F2 below = fma(F2(at_least(root[j].x(), least), at_least(root[j].y(), least)), inverse_root, eps);
        // m / below: the approximate quotient corrected by what it leaves (the division's bits for all of 2^24 drawn pairs)
        const F2 over(rcp_fast(below.x()), rcp_fast(below.y())), near = mul(m[j], over);
        const F2 p = fma(fma(fma(mul(near, minus), below, m[j]), over, near), rate, mul(F2(r.p[2 * j], r.p[2 * j + 1]), kept));
        r.p[2 * j] = p.x(), r.p[2 * j + 1] = p.y();
        // (elements behind the tensor's end are zeros)
        top_m = top_of(m[j].x(), m[j].y(), top_m);
        top_v = top_of(root[j].x(), root[j].y(), top_v);
    }
    if (x.flags & kParamBf16) store8<WIDE>(r.p, static_cast<__nv_bfloat16 *>(x.param) + at, lane, left);
    else store8<WIDE>(r.p, static_cast<float *>(x.param) + at, lane, left);
    if (x.copy) store8<WIDE>(r.p, x.copy + at, lane, left);
    // sizes as unsigned integers order as the sizes do, with a NaN above them all
    const float tm = __uint_as_float(warp_top(__float_as_uint(top_m))), tv = __uint_as_float(warp_top(__float_as_uint(top_v)));
    // Below 2^-110 a block's states are zeros: 448 / top would leave float32. (A value that rounding brings above 448 stays
    // below what the largest random number lifts to the next code, and its square's share below the smallest's.)
    const F2 im = both(tm < 0x1p-110f ? 0.f : from_top(tm)), iv = both(tv < 0x1p-110f ? 0.f : from_top(tv));
    if (lane == 0)
        *reinterpret_cast<float2 *>(x.scales + at / kBlock * 2) =
            make_float2(tm < 0x1p-110f ? 0.f : to_top(tm), tv < 0x1p-110f ? 0.f : to_top(tv));
    const uint32_t first = ((uint32_t)at + (WIDE ? lane * 8 : lane)) * kStride + start;
    uint32_t cm[8], cv[8], sign[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const F2 down = mul(mul(m[j], im), both(kDown)), value = mul(root[j], iv), bits = mul(value, both(kDown));
        const uint32_t h[2] = {mix(first + (uint32_t)(WIDE ? 2 * j : j * 64) * kStride), mix(first + (uint32_t)(WIDE ? 2 * j + 1 : j * 64 + 32) * kStride)};
        const uint32_t low[2] = {__float_as_uint(bits.x()) & 0xfff00000u, __float_as_uint(bits.y()) & 0xfff00000u};
        // v: its share of the way between the neighbours' squares against the word's upper half
        const F2 l = mul(F2(__uint_as_float(low[0]), __uint_as_float(low[1])), both(kUp)),
                 u = mul(F2(__uint_as_float(low[0] + 0x100000u), __uint_as_float(low[1] + 0x100000u)), both(kUp));
        const F2 above = mul(fma(l, minus, value), add(value, l)), step = mul(fma(l, minus, u), add(u, l));
        const F2 random = add(F2(__uint_as_float(0x3f800000u | (h[0] >> 9 & 0x7fff80u)), __uint_as_float(0x3f800000u | (h[1] >> 9 & 0x7fff80u))), both(-(1.f - 0x1p-17f)));
        const F2 border = mul(random, step);
        const float b[2] = {border.x(), border.y()}, q[2] = {above.x(), above.y()}, d[2] = {down.x(), down.y()};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            cv[2 * j + e] = (b[e] < q[e] ? low[e] + 0x100000u : low[e]) >> 20;
            // m: the upper neighbour where the word's mixed lower half, as a number in (0, 1), is below its share
            sign[2 * j + e] = __float_as_uint(d[e]);
            cm[2 * j + e] = (sign[2 * j + e] + 7u + 16u * (~(h[e] ^ h[e] >> 16) & 0xffffu)) >> 20;
        }
    }
    uint32_t qm[2], qv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        qm[i] = low_bytes(cm[4 * i], cm[4 * i + 1], cm[4 * i + 2], cm[4 * i + 3]) |
                (high_bytes(sign[4 * i], sign[4 * i + 1], sign[4 * i + 2], sign[4 * i + 3]) & 0x80808080u);
        qv[i] = low_bytes(cv[4 * i], cv[4 * i + 1], cv[4 * i + 2], cv[4 * i + 3]);
    }
    store_codes<WIDE>(qm, static_cast<uint8_t *>(x.m) + at, lane, left);
    store_codes<WIDE>(qv, static_cast<uint8_t *>(x.v) + at, lane, left);
}

// A block's run of turns, and the tensor it is in.
struct Run {
    const Tensor *tensors;
    int32_t turn, end, i, next;        // this turn, behind the last; its tensor, the next tensor's first turn
    Tensor x;
    __device__ __forceinline__ explicit Run(const Step &s) {
        tensors = reinterpret_cast<const Tensor *>(s.plan + kTensorsAt);
        const int64_t n = s.turns - s.turn;
        turn = s.turn + (int32_t)(n * blockIdx.x / gridDim.x);
        end = s.turn + (int32_t)(n * (blockIdx.x + 1) / gridDim.x);
        next = turn;
        if (turn < end) enter(reinterpret_cast<const int32_t *>(tensors + s.tensors)[turn / 2]);
    }
    __device__ __forceinline__ void enter(int32_t to) {
        i = to;
        x = tensors[i];
        next = 2 * (x.first + (int32_t)((x.n + kChunk - 1) / kChunk));
    }
    // Where the block's part of this tensor starts and ends (a last half chunk may be empty).
    __device__ __forceinline__ int64_t first() const { return (int64_t)(turn - 2 * x.first) * kTurn; }
    __device__ __forceinline__ int64_t stop() const { return min(x.n, (int64_t)(min(end, next) - 2 * x.first) * kTurn); }
    // To the next tensor.
    __device__ __forceinline__ void advance() {
        turn = min(end, next);
        if (turn < end) {
            do enter(i + 1);
            while (turn >= next);      // tensors without elements have no chunk
        }
    }
};

// Pieces of 256 elements with states in 8 bits on their way through shared memory: every lane fetches, and reads,
// its own 8 elements, so that nothing but its own copies is waited for, and no registers are held meanwhile.
constexpr int kPieces = 4;             // of a warp: one worked on, three on their way
constexpr int kPieceBytes = kThreads * 80;
struct Pieces {
    uint32_t at;                       // this thread's place in the first piece
    __device__ __forceinline__ explicit Pieces(const uint8_t *smem) : at(tc::smem_addr(smem)) {}
    // g, p: 32 bytes a thread (16 used of bfloat16), in two halves; m, v: 8
    __device__ __forceinline__ uint32_t place(int piece, int kind) const {
        return at + piece * kPieceBytes + (kind < 4 ? (kind * kThreads + threadIdx.x) * 16 : kThreads * 64 + ((kind - 4) * kThreads + threadIdx.x) * 8);
    }
    __device__ __forceinline__ void copy16(int piece, int kind, const void *from) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place(piece, kind)), "l"(from) : "memory");
    }
    __device__ __forceinline__ void copy8(int piece, int kind, const void *from) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(place(piece, kind)), "l"(from) : "memory");
    }
    __device__ __forceinline__ void fetch(int piece, const Tensor &x, uint64_t grad, int64_t first, int64_t stop) {
        const int64_t e = first + (threadIdx.x & 31) * 8;
        if (first < stop && e < x.n) {
            if (grad & 1) {
                copy16(piece, 0, reinterpret_cast<const uint16_t *>(grad - 1) + e);
            } else {
                copy16(piece, 0, reinterpret_cast<const float *>(grad) + e);
                copy16(piece, 1, reinterpret_cast<const float *>(grad) + e + 4);
            }
            if (x.flags & kParamBf16) {
                copy16(piece, 2, static_cast<const uint16_t *>(x.param) + e);
            } else {
                copy16(piece, 2, static_cast<const float *>(x.param) + e);
                copy16(piece, 3, static_cast<const float *>(x.param) + e + 4);
            }
            copy8(piece, 4, static_cast<const uint8_t *>(x.m) + e);
            copy8(piece, 5, static_cast<const uint8_t *>(x.v) + e);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ uint4 read16(int piece, int kind) const {
        uint4 r;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(place(piece, kind)) : "memory");
        return r;
    }
    __device__ __forceinline__ void eight(float (&v)[8], int piece, int kind, bool bf) const {
        const uint4 r = read16(piece, kind);
        if (bf) {
            Lot<__nv_bfloat16, 8> q;
            q.r = r;
            q.get(v);
        } else {
            const uint4 t = read16(piece, kind + 1);
            v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
            v[4] = __uint_as_float(t.x), v[5] = __uint_as_float(t.y), v[6] = __uint_as_float(t.z), v[7] = __uint_as_float(t.w);
        }
    }
    __device__ __forceinline__ void take(Share<true> &r, int piece, const Tensor &x, uint64_t grad, int64_t first) const {
        r.left = (int)min((int64_t)kBlock, x.n - first);
        if ((threadIdx.x & 31) * 8 < r.left) {
            eight(r.g, piece, 0, grad & 1);
            eight(r.p, piece, 2, x.flags & kParamBf16);
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.qm[0]), "=r"(r.qm[1]) : "r"(place(piece, 4)) : "memory");
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.qv[0]), "=r"(r.qv[1]) : "r"(place(piece, 5)) : "memory");
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) r.g[j] = r.p[j] = 0.f;
            r.qm[0] = r.qm[1] = r.qv[0] = r.qv[1] = 0;
        }
    }
};

// The values that depend on the step: the norm from the sums of squares in order, the powers of the betas.
__device__ void scalars(Scalars &shared, const Step &s, double *part) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const double *sums = reinterpret_cast<const double *>(s.plan + kSumsAt);
    double sum = 0.0;
    for (int i = threadIdx.x; i < s.sums; i += kThreads) sum += sums[i];
    if (s.sums) {
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) part[warp] = sum;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const int64_t t = *s.step + 1;
        Scalars c;
        c.factor = 1.f;
        if (s.sums) {
            sum = 0.0;
            for (int i = 0; i < kThreads / 32; ++i) sum += part[i];
            const float norm = (float)sqrt(sum);
            if (norm > s.max_norm) c.factor = __fdiv_rn(s.max_norm, norm);
            if (blockIdx.x == 0 && s.norm) *s.norm = norm;
        }
        c.lr = s.lr_at ? *s.lr_at : s.lr;
        c.rate = __fdiv_rn(c.lr, rest_of_power((float)t, s.log1_hi, s.log1_lo));
        c.inverse_root = __fdiv_rn(1.f, sqrtf(rest_of_power((float)t, s.log2_hi, s.log2_lo)));
        c.start = mixed((uint32_t)t * kStride + s.seed);
        shared = c;
        if (s.last) {        // the block that reads the step last moves it on
            Header *h = reinterpret_cast<Header *>(s.plan);
            __threadfence();
            if (atomicAdd(&h->ticket, 1u) == gridDim.x - 1) {
                h->ticket = 0;
                *s.step = t;
            }
        }
    }
    __syncthreads();
}

template <bool EIGHT>
__global__ void __launch_bounds__(kThreads, resident(EIGHT)) adamw_kernel(const __grid_constant__ Step s, const __grid_constant__ Grads grads) {
    extern __shared__ __align__(16) uint8_t queue[];
    __shared__ Scalars shared;
    __shared__ double part[kThreads / 32];
    pdl_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(2 * kTurn == kChunk && kTurn == kThreads / 32 * kBlock, "a warp's turn is 256 elements");
    Scalars c;
    bool known = false;
    auto know = [&] {              // while the first elements are on their way
        if (known) return;
        scalars(shared, s, part);
        c = shared;
        known = true;
    };
    for (Run r(s); r.turn < r.end; r.advance()) {
        int64_t at = r.first() + warp * kBlock;
        const int64_t stop = r.stop();
        const uint64_t grad = grads.at[r.i - s.first];
        if (!grad) continue;
        const bool wide = (r.x.flags & kWide) && (grad & 1 ? grad % 16 == 1 : grad % 32 == 0);
        if constexpr (EIGHT) {
            if (wide) {
                Pieces pieces(queue);
                for (int k = 0; k < kPieces - 1; ++k) pieces.fetch(k, r.x, grad, at + k * kTurn, stop);
                know();
                const uint32_t start = mixed(c.start + (uint32_t)r.i);
                auto scale_at = [&](int64_t to) {
                    return to < stop ? *reinterpret_cast<const float2 *>(r.x.scales + to / kBlock * 2) : make_float2(0.f, 0.f);
                };
                float2 scale = scale_at(at);
                int piece = 0, last = kPieces - 1;
                for (; at < stop; at += kTurn) {
                    pieces.fetch(last, r.x, grad, at + (kPieces - 1) * kTurn, stop);
                    const float2 next = scale_at(at + kTurn);
                    asm volatile("cp.async.wait_group %0;" ::"n"(kPieces - 1) : "memory");
                    Share<true> e;
                    e.scale = scale;
                    pieces.take(e, piece, r.x, grad, at);
                    update<true>(e, r.x, at, lane, c, s, start);
                    scale = next;
                    last = piece;
                    piece = piece + 1 == kPieces ? 0 : piece + 1;
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                continue;
            }
        }
        // every warp comes here equally often: the first time, all of them for the step's values
        for (bool first = true; first || at < stop; first = false, at += kTurn) {
            const bool here = at < stop;
            Share<EIGHT> e;
            if (here) wide ? load<EIGHT, true>(e, r.x, grad, at, lane) : load<EIGHT, false>(e, r.x, grad, at, lane);
            know();
            const uint32_t start = mixed(c.start + (uint32_t)r.i);
            if (here) wide ? update<true>(e, r.x, at, lane, c, s, start) : update<false>(e, r.x, at, lane, c, s, start);
        }
    }
    if (!known) scalars(shared, s, part);
}

// Sum of squares of a block's chunks; `to` says where in the table.
__global__ void __launch_bounds__(kThreads) adamw_norm_kernel(const __grid_constant__ Step s, const __grid_constant__ Grads grads, int32_t to) {
    __shared__ double part[kThreads / 32];
    pdl_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double sum = 0.0;
    for (Run r(s); r.turn < r.end; r.advance()) {
        int64_t at = r.first() + warp * kBlock;
        const int64_t stop = r.stop();
        const uint64_t grad = grads.at[r.i - s.first];
        if (!grad) continue;
        const bool bf = grad & 1, wide = r.x.n % 8 == 0 && (bf ? grad % 16 == 1 : grad % 32 == 0);
        constexpr int kAtOnce = 4;
        for (; at < stop; at += kAtOnce * kTurn) {
            float g[kAtOnce][8];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int left = (int)max((int64_t)0, min((int64_t)kBlock, stop - (at + k * kTurn)));
                if (bf) {
                    const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(grad - 1) + at + k * kTurn;
                    wide ? load8<true>(g[k], q, lane, left) : load8<false>(g[k], q, lane, left);
                } else {
                    const float *q = reinterpret_cast<const float *>(grad) + at + k * kTurn;
                    wide ? load8<true>(g[k], q, lane, left) : load8<false>(g[k], q, lane, left);
                }
            }
            float squares = 0.f;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) squares = fmaf(g[k][j], g[k][j], squares);
            sum += (double)squares;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) sum += part[i];
    reinterpret_cast<double *>(s.plan + kSumsAt)[to + blockIdx.x] = sum;
}

dendsn_status check(const dendsn_adamw_config *c) {
    if (!c) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (!std::isfinite(c->lr) || !(c->beta1 >= 0 && c->beta1 < 1) || !(c->beta2 >= 0 && c->beta2 < 1) ||
        !(c->eps >= 0 && std::isfinite(c->eps)) || !(c->max_norm >= 0 && std::isfinite(c->max_norm)))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "lr must be finite, the betas in [0, 1), eps and max_norm finite and not negative");
    if (c->state != DENDSN_STATE_F32 && c->state != DENDSN_STATE_E4M3) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown state");
    return DENDSN_OK;
}

int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_adamw_plan(const dendsn_adamw_config *cfg, const dendsn_adamw_tensor *tensors, int32_t count, void *table, size_t *table_bytes) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    if (count < 0 || (count && !tensors)) return seq_fail(DENDSN_ERR_INVALID_ARG, "tensors is NULL or count negative");
    const bool eight = cfg->state == DENDSN_STATE_E4M3;
    const size_t ss = eight ? 1 : 4;
    int64_t chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        const dendsn_adamw_tensor &t = tensors[i];
        if (t.n < 0 || (t.param_dtype != DENDSN_F32 && t.param_dtype != DENDSN_BF16) || !std::isfinite(t.weight_decay))
            return seq_fail(DENDSN_ERR_INVALID_ARG, "tensor %d: n negative, unknown param_dtype or weight_decay not finite", i);
        if (t.n && (!t.param || !t.m || !t.v || (eight && !t.scales)))
            return seq_fail(DENDSN_ERR_INVALID_ARG, "tensor %d: param, m, v or scales is NULL", i);
        if (!seq_aligned(t.param, t.param_dtype == DENDSN_BF16 ? 2 : 4) || !seq_aligned(t.m, ss) || !seq_aligned(t.v, ss) ||
            !seq_aligned(t.scales, 8) || !seq_aligned(t.copy, 2))
            return seq_fail(DENDSN_ERR_MISALIGNED, "tensor %d: param, m, v, scales (8 bytes) or copy misaligned", i);
        chunks += chunks_of(t.n);
    }
    if (chunks > INT32_MAX / 2) return seq_fail(DENDSN_ERR_UNSUPPORTED, "more than 2^30 chunks of %d elements", kChunk);
    if (table_bytes) *table_bytes = kTensorsAt + (size_t)count * sizeof(Tensor) + (size_t)chunks * 4;
    if (!table) return DENDSN_OK;
    if (!seq_aligned(table, 8)) return seq_fail(DENDSN_ERR_MISALIGNED, "table must be 8-byte aligned");
    uint8_t *to = static_cast<uint8_t *>(table);
    std::fill(to, to + kTensorsAt, (uint8_t)0);
    Tensor *x = reinterpret_cast<Tensor *>(to + kTensorsAt);
    int32_t *of = reinterpret_cast<int32_t *>(x + count);
    int32_t first = 0;
    for (int32_t i = 0; i < count; ++i) {
        const dendsn_adamw_tensor &t = tensors[i];
        const bool bf = t.param_dtype == DENDSN_BF16;
        const bool wide = t.n % 8 == 0 && seq_aligned(t.param, bf ? 16 : 32) && seq_aligned(t.m, 8 * ss) && seq_aligned(t.v, 8 * ss) && seq_aligned(t.copy, 16);
        x[i] = Tensor{t.param, t.m, t.v, t.scales, static_cast<__nv_bfloat16 *>(t.copy), t.n, first,
                      (bf ? kParamBf16 : 0) | (wide ? kWide : 0), (float)t.weight_decay, 0};
        const int32_t end = first + (int32_t)chunks_of(t.n);
        for (; first < end; ++first) of[first] = i;
    }
    return DENDSN_OK;
}

dendsn_status dendsn_adamw_step(const dendsn_adamw_config *cfg, void *plan, const int64_t *sizes, int32_t count, const void *const *grads,
                                const int32_t *grad_dtypes, int64_t *step, const float *lr, float *norm, void *stream) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    if (count < 0 || (count && (!sizes || !grads || !grad_dtypes))) return seq_fail(DENDSN_ERR_INVALID_ARG, "sizes, grads or grad_dtypes is NULL or count negative");
    if (!plan || !step) return seq_fail(DENDSN_ERR_INVALID_ARG, "plan or step is NULL");
    if (!seq_aligned(plan, 16) || !seq_aligned(step, 8) || !seq_aligned(lr, 4) || !seq_aligned(norm, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "plan (16 bytes), step, lr or norm misaligned");
    for (int32_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || (grad_dtypes[i] != DENDSN_F32 && grad_dtypes[i] != DENDSN_BF16))
            return seq_fail(DENDSN_ERR_INVALID_ARG, "tensor %d: size negative or unknown grad_dtype", i);
        if (!seq_aligned(grads[i], grad_dtypes[i] == DENDSN_BF16 ? 2 : 4))
            return seq_fail(DENDSN_ERR_MISALIGNED, "tensor %d: gradient misaligned", i);
    }
    const bool clip = cfg->max_norm > 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    Step a = {};
    a.plan = static_cast<uint8_t *>(plan);
    a.step = step;
    a.lr_at = lr;
    a.norm = norm;
    a.tensors = count;
    a.lr = (float)cfg->lr;
    a.eps = (float)cfg->eps;
    a.max_norm = (float)cfg->max_norm;
    a.rest1 = (float)(1.0 - cfg->beta1);
    a.rest2 = (float)(1.0 - cfg->beta2);
    // the logarithm of a beta of 0 as one whose power is 0 from the first step on
    const double l1 = cfg->beta1 > 0 ? std::log(cfg->beta1) : -1e4, l2 = cfg->beta2 > 0 ? std::log(cfg->beta2) : -1e4;
    a.log1_hi = (float)l1, a.log1_lo = (float)(l1 - (double)a.log1_hi);
    a.log2_hi = (float)l2, a.log2_lo = (float)(l2 - (double)a.log2_hi);
    a.seed = cfg->seed;
    const int rounds = std::max(1, (count + kGrads - 1) / kGrads);
    // blocks of each launch: the sums of squares of all launches have to fit the table
    const int most = std::max(1, kMostBlocks / rounds);
    if (clip && rounds > kMostBlocks) return seq_fail(DENDSN_ERR_UNSUPPORTED, "clipping over more than %d tensors", kGrads * kMostBlocks);
    Grads g;
    int launches = 0;
    cudaError_t e = cudaSuccess;
    for (int pass = clip ? 0 : 1; pass < 2 && e == cudaSuccess; ++pass) {
        int32_t chunk = 0;
        int sums = 0;
        for (int r = 0; r < rounds && e == cudaSuccess; ++r) {
            a.first = r * kGrads;
            a.turn = 2 * chunk;
            const int32_t end = std::min(count, a.first + kGrads);
            for (int32_t i = a.first; i < end; ++i) {
                g.at[i - a.first] = grads[i] ? reinterpret_cast<uint64_t>(grads[i]) + (grad_dtypes[i] == DENDSN_BF16 ? 1 : 0) : 0;
                chunk += (int32_t)chunks_of(sizes[i]);
            }
            a.turns = 2 * chunk;
            a.last = r == rounds - 1;
            const int blocks = std::max(1, std::min(a.turns - a.turn, pass ? 152 * resident(cfg->state == DENDSN_STATE_E4M3) : most));
            if (pass == 0) {
                e = seq_launch(adamw_norm_kernel, dim3((unsigned)blocks), kThreads, 0, s, 1, a, g, sums);
                sums += blocks;
            } else {
                if (cfg->state == DENDSN_STATE_E4M3) {
                    constexpr int kBytes = kPieces * kPieceBytes;
                    e = cudaFuncSetAttribute(adamw_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
                    if (e == cudaSuccess) e = seq_launch(adamw_kernel<true>, dim3((unsigned)blocks), kThreads, kBytes, s, 1, a, g);
                } else {
                    e = seq_launch(adamw_kernel<false>, dim3((unsigned)blocks), kThreads, 0, s, 1, a, g);
                }
            }
            ++launches;
        }
        if (pass == 0) a.sums = sums;
    }
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "adamw launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(launches);
    return DENDSN_OK;
}

}  // extern "C"
