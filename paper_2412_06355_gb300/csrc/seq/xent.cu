// Softmax cross entropy of a linear readout in pieces of the vocabulary, and its gradient.
//
// Four products, all on the fifth-generation tensor cores (tcgen05 on a pair of blocks, a
// 256 x 256 tile of float32 sums in TMEM, operands by tensor copies into 128-byte-swizzled
// shared memory):
//   STATS   l = H W^T of all the vocabulary; the epilogue keeps each row's maximum and sum of
//           exponentials of 128 columns, and the label's logit; a small kernel joins them
//   PIECE   l again for one piece of the vocabulary; the epilogue writes
//           G = c (exp(l - lse) - [label]) as bfloat16 terms
//   HIDDEN  grad_hidden += G W of the piece, in float32
//   WEIGHT  grad_weight of the piece = G^T H
// so 2 M V D operations in the forward; in the backward 10 M V D for bfloat16 operands with G in
// two terms (6 M V D with G rounded to one, which the caller may choose), of which 2 M V D form the
// logits again instead of keeping M V of them. Forward and backward of 8192 rows, V = 131072, D = 2048
// take 10.4 ms with G in one term and 15.4 ms in two; the error of the gradients against 64 bits is
// 2.4e-3 and 1.7e-3, that of rounding the exact gradients. Bound by the tensor cores: that size takes
// 2.36-2.41 ms forward and 12.8 ms backward (1.7-1.8 PFLOP/s) under the card's power limit, where cuBLAS
// sustains 1.75; 4096 rows, V = 50000, D = 1024: 228 and 1270 us. Few rows are bound by reading
// the weights and by three launches (16 rows, V = 32768, D = 384: 16 us).
//
// The logits are float32 sums of the tensor core, which loses more than float32 additions do: the
// loss of bfloat16 operands is off by 4.0e-8 of itself at D = 64, 1.3e-7 at 384, 7.7e-7 at 2048, where
// float32 additions leave 4.0e-8, 4.4e-8 and 8.0e-8. Adding the sums to registers every 256 terms,
// as is done for float32 operands, gives 8.7e-8 and costs the forward 27% at D = 1024: not done.
//
// Rows that are ignored are left out before the products: the others are copied together
// (xent_rows, xent_pack), so ignored rows cost nothing and no infinity or NaN in them can
// reach a product as 0 * inf. That copy also gives rows of any D the 16-byte pitch that
// tensor copies need, and float32 operands their three bfloat16 terms: x = x0 + x1 + x2 with
// 8 bits each; the products x_i y_j with i + j <= 2 are summed, the smallest first, and the
// others are at most 2^-24 of x y together.
#include <cuda_bf16.h>

#include <algorithm>
#include <mutex>

#include "pairs.cuh"
#include "seq_common.h"
#include "tc.cuh"

namespace dendsn {
namespace {

enum { STATS = 0, PIECE = 1, HIDDEN = 2, WEIGHT = 3 };

constexpr int kTileM = 256, kTileN = 256, kTileK = 64;    // of a pair of blocks
constexpr int kStages = 6;
// float32 operands: blocks of the sum after which the tile's sums in TMEM are added to float32
// registers and begin anew. The tensor core's running sums lose more than a float32 addition
// does (in one run over 10,007 terms the relative error of grad_hidden was 1.5e-6).
constexpr int kChunk = 4;
constexpr int kHalfBytes = 128 * kTileK * 2;              // one block's 128 x 64 operand tile
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kThreads = 320;                             // copies, products, 8 warps of epilogue
constexpr size_t kSmem = kStages * kStageBytes + 1024 + 256;
constexpr int kIgnored = -1, kBadLabel = -2;
constexpr float kLog2e = 1.4426950408889634f;

struct Ctl {                // at the start of the scratch buffer
    int32_t rows;           // rows that take part
    int32_t failed;         // a wait ran out: results become NaN
    int32_t pad[62];
};

template <typename I>
__device__ __forceinline__ int label_of(const void *labels, int64_t r, int V, int64_t ignore) {
    const int64_t y = static_cast<const I *>(labels)[r];
    return y == ignore ? kIgnored : (y < 0 || y >= V) ? kBadLabel : (int)y;
}
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

__device__ __forceinline__ uint32_t two(__nv_bfloat16 a, __nv_bfloat16 b) {
    return (uint32_t)__bfloat16_as_ushort(a) | (uint32_t)__bfloat16_as_ushort(b) << 16;
}

// The terms of x = x0 + x1 + x2, each the rounding of what the ones before it leave. A finite x whose
// rounding would overflow is truncated; what is not finite stays in the first term alone.
__device__ __forceinline__ void split(float x, __nv_bfloat16 (&t)[3]) {
    t[0] = __float2bfloat16_rn(x);
    if (!isfinite(__bfloat162float(t[0]))) {
        if (!isfinite(x)) {
            t[1] = t[2] = __float2bfloat16_rn(0.f);
            return;
        }
        t[0] = __float2bfloat16_rz(x);
    }
    const float r = x - __bfloat162float(t[0]);
    t[1] = __float2bfloat16_rn(r);
    t[2] = __float2bfloat16_rn(r - __bfloat162float(t[1]));
}

// The second of two terms x = x0 + x1 (within 2^-16 of x); none where x0 is not finite.
__device__ __forceinline__ __nv_bfloat16 remainder_of(float x, __nv_bfloat16 first) {
    const float f = __bfloat162float(first);
    return __float2bfloat16_rn(isfinite(f) ? x - f : 0.f);
}

// ------------------------------------------------------------------ rows that take part
struct Rows {
    Ctl *ctl;
    int32_t *index;         // [Mp] row of the call
    int32_t *label;         // [Mp]
    int32_t *where;         // [M] place of a row, or kIgnored, kBadLabel
    float *lse, *scale, *weight;   // [Mp] of the backward: G = scale exp(l - lse), minus weight at the label
    float *picked;          // [Mp] of the forward: the label's logit
};

// Per-row inputs and outputs that the list of rows takes along. lse_sum: the second row of
// statistics, the sums beside the maxima in lse, or null where lse is one number.
struct PerRow {
    const void *labels;
    float *loss, *lse_out, *sum_out;              // of the forward: written for rows that do not take part
    const float *lse, *lse_sum, *gloss;           // of the backward
};
__device__ __forceinline__ void leave_out(const PerRow &p, int64_t r, int y) {
    const float v = y == kIgnored ? 0.f : nan_f();
    p.loss[r] = p.lse_out[r] = v;
    if (p.sum_out) p.sum_out[r] = v;
}
__device__ __forceinline__ void take_along(const Rows &R, const PerRow &p, int at, int64_t r) {
    const float w = p.gloss[r];
    R.lse[at] = p.lse[r];
    R.scale[at] = p.lse_sum ? w / p.lse_sum[r] : w;
    R.weight[at] = w;
}

// One block: lists the rows with a label in the vocabulary, in order, and fills the places up
// to the next multiple of 256 with rows of weight zero.
template <typename I>
__global__ void __launch_bounds__(1024) xent_rows_kernel(Rows R, PerRow p, int32_t M, int32_t V, int64_t ignore) {
    pdl_begin();
    constexpr int kEach = 8;                                  // consecutive rows of a thread
    __shared__ int warps[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int done = 0;
    for (int64_t r0 = 0; r0 < M; r0 += 1024 * kEach) {
        const int64_t r = r0 + threadIdx.x * kEach;
        int y[kEach], mine = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) y[j] = r + j < M ? label_of<I>(p.labels, r + j, V, ignore) : kIgnored;
#pragma unroll
        for (int j = 0; j < kEach; ++j) mine += y[j] >= 0;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) warps[warp] = incl;
        __syncthreads();
        int at = done + incl - mine;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) at += warps[w];
            done += warps[w];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (r + j >= M) break;
            R.where[r + j] = y[j] >= 0 ? at : y[j];
            if (y[j] >= 0) {
                R.index[at] = (int32_t)(r + j);
                R.label[at] = y[j];
                if (p.lse) take_along(R, p, at, r + j);
                ++at;
            } else if (p.loss) {
                leave_out(p, r + j, y[j]);
            }
        }
    }
    const int end = (done + kTileM - 1) / kTileM * kTileM;
    for (int i = done + threadIdx.x; i < end; i += 1024) {
        R.index[i] = -1;
        R.label[i] = -1;
        if (p.lse) R.lse[i] = R.scale[i] = R.weight[i] = 0.f;
    }
    if (threadIdx.x == 0) {
        R.ctl->rows = done;
        R.ctl->failed = 0;
    }
}

// Copies a row of D elements (none: zeros) to Dp bfloat16 elements with zeros behind, in three
// planes for float32; a thread of the warp takes 8 elements at a time. WIDE: rows can be read 16
// bytes at a time.
template <typename T, bool WIDE>
__device__ __forceinline__ void pack_row(const T *p, __nv_bfloat16 *to, int lane, int32_t D, int32_t Dp, int64_t plane) {
    for (int32_t d = lane * 8; d < Dp; d += 256) {
        uint4 *q = reinterpret_cast<uint4 *>(to + d);
        if constexpr (sizeof(T) == 2) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if (p) {
                if (WIDE) {
                    if (d < D) w = __ldg(reinterpret_cast<const uint4 *>(p + d));
                } else {
                    __nv_bfloat16 e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = d + j < D ? p[d + j] : __float2bfloat16_rn(0.f);
                    w = make_uint4(two(e[0], e[1]), two(e[2], e[3]), two(e[4], e[5]), two(e[6], e[7]));
                }
            }
            *q = w;
        } else {
            float e[8] = {};
            if (p) {
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    if (WIDE) {
                        if (d + h < D) {
                            const float4 f = __ldg(reinterpret_cast<const float4 *>(p + d + h));
                            e[h] = f.x;
                            e[h + 1] = f.y;
                            e[h + 2] = f.z;
                            e[h + 3] = f.w;
                        }
                    } else {
#pragma unroll
                        for (int j = h; j < h + 4; ++j) e[j] = d + j < D ? p[d + j] : 0.f;
                    }
                }
            }
            uint32_t w[3][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                __nv_bfloat16 u[3], v[3];
                split(e[2 * j], u);
                split(e[2 * j + 1], v);
#pragma unroll
                for (int t = 0; t < 3; ++t) w[t][j] = two(u[t], v[t]);
            }
#pragma unroll
            for (int t = 0; t < 3; ++t) q[t * (plane / 8)] = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
        }
    }
}

// index: the row to copy for each place (negative: zeros), or null: the same row.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) xent_pack_kernel(const T *from, __nv_bfloat16 *to, const int32_t *index,
                                                        const Ctl *ctl, int64_t rows, int32_t D, int32_t Dp,
                                                        int64_t plane) {
    pdl_begin();
    const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (r >= rows) return;
    int64_t src = r;
    if (index) {
        if (r >= (ctl->rows + kTileM - 1) / kTileM * kTileM) return;
        src = index[r];
    }
    pack_row<T, WIDE>(src >= 0 ? from + src * D : nullptr, to + r * Dp, threadIdx.x & 31, D, Dp, plane);
}

// xent_rows and xent_pack of the hidden rows in one launch, for up to kFewRows rows: every block
// lists the rows for itself, block 0 writes the list down, and each warp copies one place.
constexpr int kFewRows = 1024;

template <typename T, typename I, bool WIDE>
__global__ void __launch_bounds__(256) xent_rows_pack_kernel(Rows R, PerRow p, int32_t M, int32_t V, int64_t ignore,
                                                             const T *from, __nv_bfloat16 *to, int32_t D, int32_t Dp,
                                                             int64_t plane) {
    pdl_begin();
    constexpr int kEach = kFewRows / 256;
    __shared__ int warps[8], list[kFewRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r0 = threadIdx.x * kEach;
    int y[kEach], mine = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        y[j] = r0 + j < M ? label_of<I>(p.labels, r0 + j, V, ignore) : kIgnored;
        mine += y[j] >= 0;
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) warps[warp] = incl;
    __syncthreads();
    int at = incl - mine, rows = 0;
    for (int w = 0; w < 8; ++w) {
        if (w < warp) at += warps[w];
        rows += warps[w];
    }
    const int end = (rows + kTileM - 1) / kTileM * kTileM;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int r = r0 + j;
        if (r >= M) break;
        if (y[j] >= 0) list[at] = r;
        if (blockIdx.x == 0) {
            R.where[r] = y[j] >= 0 ? at : y[j];
            if (y[j] >= 0) {
                R.index[at] = r;
                R.label[at] = y[j];
                if (p.lse) take_along(R, p, at, r);
            } else if (p.loss) {
                leave_out(p, r, y[j]);
            }
        }
        at += y[j] >= 0;
    }
    if (blockIdx.x == 0) {
        for (int i = rows + threadIdx.x; i < end; i += 256) {
            R.index[i] = R.label[i] = -1;
            if (p.lse) R.lse[i] = R.scale[i] = R.weight[i] = 0.f;
        }
        if (threadIdx.x == 0) {
            R.ctl->rows = rows;
            R.ctl->failed = 0;
        }
    }
    __syncthreads();
    const int place = blockIdx.x * 8 + warp;
    if (place < end)
        pack_row<T, WIDE>(place < rows ? from + (int64_t)list[place] * D : nullptr, to + (int64_t)place * Dp, lane, D, Dp, plane);
}

// ------------------------------------------------------------------ the products
struct Gemm {
    Ctl *ctl;
    const int32_t *label;
    const float *lse, *scale, *weight;
    float *picked;
    float2 *part;           // [2 * nt][Mp]
    __nv_bfloat16 *G;       // [gterms][Mp][pitch]
    float *sum;             // [splits][Mp][nt * kTileN]
    void *gw;               // [V][D]
    int64_t Mp, gplane;
    int32_t pitch;
    int32_t mt, nt, splits; // tiles (mt of the products over rows follows from ctl->rows)
    int32_t kb, kb_split;   // blocks of kTileK along the sum, in all and for one split
    int32_t gterms;         // of G
    int32_t V, D, v0, vc;
    bool wide;              // rows of gw can be written 32 bytes at a time
};

// The operand terms of each pass over the sum, smallest products first.
__device__ __forceinline__ int term_a(int phase) { return 0x201100 >> (20 - 4 * phase) & 0xf; }
__device__ __forceinline__ int term_b(int phase) { return 0x021010 >> (20 - 4 * phase) & 0xf; }

template <int MODE> __device__ __forceinline__ void tile_of(const Gemm &g, int mt, int64_t item, int &m, int &n, int &s) {
    s = 0;
    if (MODE == STATS || MODE == PIECE) {      // the hidden rows stay in L2, the weights pass once
        m = (int)(item % mt);
        n = (int)(item / mt);
    } else {                                   // G passes once
        n = (int)(item % g.nt);
        const int64_t rest = item / g.nt;
        m = (int)(rest % mt);
        s = (int)(rest / mt);
    }
}

template <int MODE, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    xent_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const Gemm g) {
    constexpr bool kF32 = sizeof(T) == 4;
    // Products of terms for each block of the sum. bfloat16 inputs have one term, their G as many
    // as the caller chose.
    const int phases = kF32 ? 6 : MODE == HIDDEN || MODE == WEIGHT ? g.gterms : 1;
    constexpr bool kRowsA = MODE != WEIGHT;                   // operand rows run along the sum
    constexpr bool kRowsB = MODE == STATS || MODE == PIECE;
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t tmem_base;
    const uint32_t stage0 = (tc::smem_addr(raw) + 1023) & ~1023u;
    const uint32_t bars = stage0 + kStages * kStageBytes;
    const uint32_t full = bars, empty = bars + 8 * kStages, acc_full = bars + 16 * kStages, acc_empty = acc_full + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_rank();
    const int64_t first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (warp == 0 && lane == 0) {
        for (int i = 0; i < kStages; ++i) {
            tc::bar_init(full + 8 * i, 1);
            tc::bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(acc_full + 8 * i, 1);
            tc::bar_init(acc_empty + 8 * i, 16);
        }
        tc::bar_init_fence();
        tc::prefetch_map(&map_a);
        tc::prefetch_map(&map_b);
    }
    if (warp == 1) tc::tmem_alloc(tc::smem_addr(&tmem_base), 512);
    tc::fence_before_sync();
    __syncthreads();
    tc::cluster_sync();
    tc::fence_after_sync();
    const uint32_t tmem = tmem_base;
    bool ok = true;
    pdl_begin();                                              // nothing before this reads or writes memory
    const int rows = g.ctl->rows;
    const int mt = MODE == WEIGHT ? g.mt : (rows + kTileM - 1) / kTileM;
    const int kb = MODE == WEIGHT ? (rows + kTileK - 1) / kTileK : g.kb;
    const int64_t items = (int64_t)mt * g.nt * g.splits;

    if (warp == 0 && lane == 0) {                             // copies, in both blocks
        const uint32_t full0 = tc::in_block(full, 0);
        int stage = 0;
        uint32_t phase = 1;
        for (int64_t item = first; ok && item < items; item += stride) {
            int m, n, s;
            tile_of<MODE>(g, mt, item, m, n, s);
            const int am = m * kTileM + (int)rank * 128, bn = n * kTileN + (int)rank * 128;
            const int k0 = s * g.kb_split, k1 = MODE == WEIGHT ? kb : min(kb, k0 + g.kb_split);
            const int chunk = kF32 ? kChunk : max(1, k1 - k0);
            for (int c0 = k0; ok && c0 < k1; c0 += chunk) {
                const int end = min(k1, c0 + chunk);
                // float32: the chunk's blocks for one product of terms after the other; bfloat16: the
                // terms of G for one block after the other, which find the other operand in L2
                for (int k = c0, ph = 0; k < end && ph < phases;) {
                    const int ta = kF32 ? term_a(ph) : phases - 1 - ph, tb = kF32 ? term_b(ph) : 0;
                    if (!(ok = tc::bar_wait(empty + 8 * stage, phase))) break;
                    if (rank == 0) tc::bar_expect(full + 8 * stage, 2 * kStageBytes);
                    const uint32_t a = stage0 + stage * kStageBytes, b = a + kHalfBytes, bar = full0 + 8 * stage;
                    if (kRowsA) {
                        tc::load_box(a, &map_a, bar, k * kTileK, am, ta);
                    } else {
                        tc::load_box(a, &map_a, bar, am, k * kTileK, ta);
                        tc::load_box(a + kHalfBytes / 2, &map_a, bar, am + 64, k * kTileK, ta);
                    }
                    if (kRowsB) {
                        tc::load_box(b, &map_b, bar, k * kTileK, g.v0 + bn, tb);
                    } else {
                        const int row = MODE == HIDDEN ? g.v0 + k * kTileK : k * kTileK;
                        tc::load_box(b, &map_b, bar, bn, row, tb);
                        tc::load_box(b + kHalfBytes / 2, &map_b, bar, bn + 64, row, tb);
                    }
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                    if (kF32) {
                        if (++k == end) { k = c0; ++ph; }
                    } else if (++ph == phases) {
                        ph = 0;
                        ++k;
                    }
                }
            }
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {         // products, in the first block
        constexpr uint32_t idesc = tc::product_of(kTileM, kTileN, !kRowsA, !kRowsB);
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 1;
        for (int64_t item = first; ok && item < items; item += stride) {
            int m, n, s;
            tile_of<MODE>(g, mt, item, m, n, s);
            const int k0 = s * g.kb_split, k1 = MODE == WEIGHT ? kb : min(kb, k0 + g.kb_split);
            const int chunk = kF32 ? kChunk : max(1, k1 - k0);
            for (int c0 = k0; ok && c0 < k1; c0 += chunk) {
                const int steps = min(chunk, k1 - c0) * phases;
                if (!(ok = tc::bar_wait(acc_empty + 8 * acc, acc_phase))) break;
                tc::fence_after_sync();
                for (int i = 0; i < steps; ++i) {
                    if (!(ok = tc::bar_wait(full + 8 * stage, phase))) break;
                    tc::fence_after_sync();
                    const uint32_t a = stage0 + stage * kStageBytes, b = a + kHalfBytes;
#pragma unroll
                    for (int j = 0; j < kTileK / 16; ++j)
                        tc::mma(tmem + acc * kTileN, tc::operand(a + j * (kRowsA ? 32 : 2048), kRowsA, kHalfBytes / 2),
                                tc::operand(b + j * (kRowsB ? 32 : 2048), kRowsB, kHalfBytes / 2), idesc, i + j > 0);
                    tc::commit_both(empty + 8 * stage);
                    if (++stage == kStages) { stage = 0; phase ^= 1; }
                }
                if (!ok) break;
                tc::commit_both(acc_full + 8 * acc);
                if (++acc == 2) { acc = 0; acc_phase ^= 1; }
            }
        }
    } else if (warp >= 2) {                                   // epilogue, in both blocks
        const int quad = warp % 4, half = (warp - 2) / 4;
        const uint32_t empty0 = tc::in_block(acc_empty, 0);
        int acc = 0;
        uint32_t acc_phase = 0;
        // what the epilogue needs of its row is requested one tile ahead
        int next_y = -1;
        float next_lse = 0.f, next_scale = 0.f, next_weight = 0.f;
        auto request = [&](int64_t item) {
            if ((MODE == STATS || MODE == PIECE) && item < items) {
                int m, n, s;
                tile_of<MODE>(g, mt, item, m, n, s);
                const int row = m * kTileM + (int)rank * 128 + quad * 32 + lane;
                next_y = g.label[row];
                if (MODE == PIECE) {
                    next_lse = g.lse[row];
                    next_scale = g.scale[row];
                    next_weight = g.weight[row];
                }
            }
        };
        request(first);
        for (int64_t item = first; item < items; item += stride) {
            int m, n, s;
            tile_of<MODE>(g, mt, item, m, n, s);
            const int k0 = s * g.kb_split, k1 = MODE == WEIGHT ? kb : min(kb, k0 + g.kb_split);
            const bool any = k1 > k0;
            const int y = next_y;
            const float lse = next_lse, scale = next_scale, weight = next_weight;
            request(item + stride);
            const int row = m * kTileM + (int)rank * 128 + quad * 32 + lane;
            const int col0 = n * kTileN + half * 128;
            // the tile's sums are in TMEM; takes them over once they are complete
            auto take = [&] {
                ok = __all_sync(0xffffffffu, tc::bar_wait(acc_full + 8 * acc, acc_phase));
                tc::fence_after_sync();
            };
            auto give_back = [&] {
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::bar_arrive_cluster(empty0 + 8 * acc);
                if (++acc == 2) { acc = 0; acc_phase ^= 1; }
            };
            auto columns = [&](int c) { return tmem + ((uint32_t)quad << 21) + acc * kTileN + half * 128 + 32 * c; };
            float sums[kF32 ? 4 : 2][32];
            if constexpr (kF32) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sums[c][i] = 0.f;
                for (int c0 = k0; c0 < k1; c0 += kChunk) {
                    take();
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v[32];
                        tc::tmem_load(v, columns(c));
#pragma unroll
                        for (int i = 0; i < 32; ++i) sums[c][i] += v[i];
                    }
                    give_back();
                }
            } else if (any) {
                take();
            }
            if (!ok) break;
            float top = -INFINITY, total = 0.f;
            auto epilogue = [&](int c, float (&v)[32]) {
                const int col = col0 + 32 * c;                // within the piece, or within D
                if (MODE == STATS) {
                    const int left = g.V - col;
                    if (left < 32)
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = i < left ? v[i] : -INFINITY;
                    if (y >= col && y < col + 32)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (y == col + i) g.picked[row] = v[i];
                    // Half an instruction an element for each of the maximum, the exponent and the
                    // sum; the exponentials themselves (16 a clock and SM) bound the epilogue.
                    float t = top;
#pragma unroll
                    for (int i = 0; i < 32; i += 2) t = max3(t, v[i], v[i + 1]);
                    // the maximum is subtracted first: the difference is exact for the terms that
                    // count, whatever the logits' size
                    const float ref = t == -INFINITY ? 0.f : t;
                    F2 sum[2] = {both(0.f), both(0.f)};
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const F2 e = mul(add(F2(v[i], v[i + 1]), both(-ref)), both(kLog2e));
                        sum[i / 2 % 2] = add(sum[i / 2 % 2], F2(exp2_fast(e.x()), exp2_fast(e.y())));
                    }
                    const F2 s2 = add(sum[0], sum[1]);
                    total = (total == 0.f ? 0.f : total * exp2_fast((top - ref) * kLog2e)) + (s2.x() + s2.y());
                    top = t;
                } else if (MODE == PIECE) {
                    // c p = scale exp(l - lse), the difference first, whose size alone decides its rounding
                    const F2 w = both(scale), base = both(-lse);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const F2 l(v[i], v[i + 1]);
                        const F2 e = mul(add(l, base), both(kLog2e));
                        const F2 p = mul(F2(exp2_fast(e.x()), exp2_fast(e.y())), w);
                        v[i] = p.x();
                        v[i + 1] = p.y();
                    }
                    const int at = y - g.v0 - col;
                    if (at >= 0 && at < 32)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i == at) v[i] -= weight;
                    __nv_bfloat16 *to = g.G + (int64_t)row * g.pitch + col;
#pragma unroll
                    for (int i = 0; i < 32; i += 16) {
                        if constexpr (!kF32) {
                            uint32_t q[8], rest[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const __nv_bfloat16 a = __float2bfloat16_rn(v[i + 2 * j]), b = __float2bfloat16_rn(v[i + 2 * j + 1]);
                                q[j] = two(a, b);
                                rest[j] = two(remainder_of(v[i + 2 * j], a), remainder_of(v[i + 2 * j + 1], b));
                            }
                            tc::store32(to + i, q);
                            if (g.gterms == 2) tc::store32(to + i + g.gplane, rest);
                        } else {
                            uint32_t q[3][8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                __nv_bfloat16 a[3], b[3];
                                split(v[i + 2 * j], a);
                                split(v[i + 2 * j + 1], b);
#pragma unroll
                                for (int t = 0; t < 3; ++t) q[t][j] = two(a[t], b[t]);
                            }
#pragma unroll
                            for (int t = 0; t < 3; ++t) tc::store32(to + i + t * g.gplane, q[t]);
                        }
                    }
                } else if (MODE == HIDDEN) {
                    float *to = g.sum + ((int64_t)s * g.Mp + row) * (g.nt * kTileN) + col;
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint32_t q[8];
                        if (g.v0) {
                            tc::load32(q, to + i);
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[i + j] += __uint_as_float(q[j]);
                        }
#pragma unroll
                        for (int j = 0; j < 8; ++j) q[j] = __float_as_uint(v[i + j]);
                        tc::store32(to + i, q);
                    }
                } else {
                    T *to = static_cast<T *>(g.gw) + ((int64_t)g.v0 + row) * g.D + col;
                    if (row < g.vc) {
                        if (g.wide && col + 32 <= g.D) {
                            constexpr int kEach = 32 / sizeof(T);
#pragma unroll
                            for (int i = 0; i < 32; i += kEach) {
                                uint32_t q[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    if constexpr (kF32) q[j] = __float_as_uint(v[i + j]);
                                    else q[j] = two(__float2bfloat16_rn(v[i + 2 * j]), __float2bfloat16_rn(v[i + 2 * j + 1]));
                                }
                                tc::store32(to + i, q);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (col + i < g.D) to[i] = from_f<T>(v[i]);
                        }
                    }
                }
            };
            if constexpr (kF32) {
#pragma unroll
                for (int c = 0; c < 4; ++c) epilogue(c, sums[c]);
            } else {
#pragma unroll 1
                for (int c = 0; c < 4; c += 2) {
                    if (any) tc::tmem_load(sums, columns(c));
                    else
#pragma unroll
                        for (int i = 0; i < 32; ++i) sums[0][i] = sums[1][i] = 0.f;
                    epilogue(c, sums[0]);
                    epilogue(c + 1, sums[1]);
                }
                if (any) give_back();
            }
            if (MODE == STATS)
                g.part[(int64_t)(2 * n + half) * g.Mp + row] = make_float2(top, total);
        }
    }
    if (!ok) g.ctl->failed = 1;
    __syncwarp();
    tc::fence_before_sync();
    // where a wait ran out, copies and products may still be on their way: they land before the
    // pair's shared memory and TMEM are given back
    if (!__syncthreads_and(ok)) let_land();
    tc::cluster_sync();
    tc::fence_after_sync();
    if (warp == 1) tc::tmem_free(tmem, 512);
}

// ------------------------------------------------------------------ few float32 rows
// The statistics of up to 32 float32 rows straight from the float32 operands: three bfloat16
// terms of all the weights would be written and read for a handful of rows (16 bytes a weight
// against 4). A block forms the logits of MT rows with 64 vocabulary rows by multiply-adds on
// pairs along the sum, 32 terms a stage copied ahead (cp.async), and keeps each row's maximum and
// sum of exponentials. A thread takes all MT rows of one or two vocabulary rows, so that every
// weight is read from shared memory once and the hidden values are broadcast; the warps share
// the terms of a stage and are added up at the end. Rows of a stage lie 36 floats apart, so that
// no two lanes of a wide read meet in a bank. Whole calls at V = 50000, D = 1024: 16 rows 81 us
// (187 in terms; 205 MB of weights would take 30), 32 rows 164 us (191); 64 rows would take 296 us (194 in
// terms), so the terms begin at 33 rows. Stages of 64 terms: 92 and 163 us.
constexpr int kFewF32 = 32, kFewV = 64, kFewK = 32, kFewPitch = kFewK + 4, kFewStages = 3;
template <int MT> constexpr size_t kFewSmem = (size_t)kFewStages * (MT + kFewV) * kFewPitch * 4;
static_assert(8 * 16 * (kFewV + 1) * 4 <= kFewSmem<16> && 4 * 32 * (kFewV + 1) * 4 <= kFewSmem<32>, "the warps' logits fit");

template <int MT, bool WIDE>
__global__ void __launch_bounds__(256) xent_few_kernel(Rows R, const float *hidden, const float *weight, float2 *part,
                                                       int32_t V, int32_t D, int64_t Mp) {
    pdl_begin();
    constexpr int kV = MT == 16 ? 2 : 1;                      // vocabulary rows of a thread
    constexpr int kVWarps = kFewV / (32 * kV), kKWarps = 8 / kVWarps;
    constexpr int kStage = (MT + kFewV) * kFewPitch;
    extern __shared__ __align__(16) float few[];
    const int rows = R.ctl->rows, v0 = blockIdx.x * kFewV;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = warp % kVWarps * 32 * kV + lane, kw = warp / kVWarps;
    const int chunks = (D + kFewK - 1) / kFewK;
    // 8 threads copy 32 terms of a row; rows beyond the operands and terms beyond D become zeros
    constexpr int kLines = 32, kW = kFewV / kLines, kH = (MT + kLines - 1) / kLines;
    const int quad = threadIdx.x % 8 * 4, line = threadIdx.x / 8;
    auto copy = [&](float *to, const float *from, bool there, int k) {
        const uint32_t dst = tc::smem_addr(to);
        if constexpr (WIDE) {
            const int bytes = there && k < D ? 16 : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(bytes ? from + k : from), "r"(bytes)
                         : "memory");
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bytes = there && k + j < D ? 4 : 0;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j),
                             "l"(bytes ? from + k + j : from), "r"(bytes) : "memory");
            }
        }
    };
    const float *w_from[kW], *h_from[kH];
    bool w_there[kW], h_there[kH];
#pragma unroll
    for (int i = 0; i < kW; ++i) {
        const int v = v0 + line + kLines * i;
        w_there[i] = v < V;
        w_from[i] = weight + (w_there[i] ? (int64_t)v * D : 0);
    }
#pragma unroll
    for (int i = 0; i < kH; ++i) {
        const int r = line + kLines * i;
        h_there[i] = r < rows;
        h_from[i] = hidden + (h_there[i] ? (int64_t)R.index[r] * D : 0);
    }
    auto fetch = [&](int chunk) {
        if (chunk < chunks) {
            float *w = few + chunk % kFewStages * kStage, *h = w + kFewV * kFewPitch;
            const int k = chunk * kFewK + quad;
#pragma unroll
            for (int i = 0; i < kW; ++i) copy(w + (line + kLines * i) * kFewPitch + quad, w_from[i], w_there[i], k);
#pragma unroll
            for (int i = 0; i < kH; ++i)
                if (line + kLines * i < MT) copy(h + (line + kLines * i) * kFewPitch + quad, h_from[i], h_there[i], k);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    F2 acc[MT][kV];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < kV; ++j) acc[i][j] = both(0.f);
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) fetch(i);
    for (int chunk = 0; chunk < chunks; ++chunk) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
        __syncthreads();                                      // the chunk is there, the one before it is read
        fetch(chunk + kFewStages - 1);
        const float *w = few + chunk % kFewStages * kStage, *h = w + kFewV * kFewPitch;
#pragma unroll
        for (int u = 0; u < kFewK; u += 4 * kKWarps) {
            const int k = u + 4 * kw;
            float4 b[kV];
#pragma unroll
            for (int j = 0; j < kV; ++j) b[j] = *reinterpret_cast<const float4 *>(w + (col + 32 * j) * kFewPitch + k);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const float4 a = *reinterpret_cast<const float4 *>(h + i * kFewPitch + k);
#pragma unroll
                for (int j = 0; j < kV; ++j)
                    acc[i][j] = fma(F2(a.z, a.w), F2(b[j].z, b[j].w), fma(F2(a.x, a.y), F2(b[j].x, b[j].y), acc[i][j]));
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    constexpr int kRow = kFewV + 1;
    float *logits = few;                                      // [kKWarps][MT][kRow]
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < kV; ++j) logits[(kw * MT + i) * kRow + col + 32 * j] = acc[i][j].x() + acc[i][j].y();
    __syncthreads();
    for (int r = warp; r < min(MT, rows); r += 8) {
        const int y = R.label[r];
        float l[2], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int v = v0 + lane + 32 * j;
            l[j] = 0.f;
#pragma unroll
            for (int k = 0; k < kKWarps; ++k) l[j] += logits[(k * MT + r) * kRow + lane + 32 * j];
            if (v >= V) l[j] = -INFINITY;
            if (v == y) R.picked[r] = l[j];
            top = fmaxf(top, l[j]);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ref = top == -INFINITY ? 0.f : top;
        float total = exp2_fast((l[0] - ref) * kLog2e) + exp2_fast((l[1] - ref) * kLog2e);
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        if (lane == 0) part[(int64_t)blockIdx.x * Mp + r] = make_float2(top, total);
    }
}

// Joins the maxima and sums of a row: 32 rows of a block, its 32 warps take every 32nd part,
// eight of them in flight.
__global__ void __launch_bounds__(1024) xent_join_kernel(Rows R, const float2 *part, int32_t parts, int64_t Mp,
                                                         float *loss, float *lse, float *sum) {
    pdl_begin();
    __shared__ float2 sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = blockIdx.x * 32 + lane;
    const int rows = R.ctl->rows;
    if (blockIdx.x * 32 >= rows) return;
    float2 a = make_float2(-INFINITY, 0.f);
    auto add = [](float2 &x, const float2 &y) {
        if (y.y == 0.f) return;                               // nothing in it
        const float m = fmaxf(x.x, y.x);
        x.y = (x.y == 0.f ? 0.f : x.y * expf(x.x - m)) + y.y * expf(y.x - m);
        x.x = m;
    };
    if (r < rows)
        for (int p = warp; p < parts; p += 256) {
            float2 q[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                q[u] = p + 32 * u < parts ? __ldg(part + (int64_t)(p + 32 * u) * Mp + r) : make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 8; ++u) add(a, q[u]);
        }
    sh[warp][lane] = a;
    __syncthreads();
    // warp w joins the 32 parts of row w, in an order that is always the same
    float2 b = sh[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float2 other = make_float2(__shfl_down_sync(0xffffffffu, b.x, o), __shfl_down_sync(0xffffffffu, b.y, o));
        add(b, other);
    }
    const int row = blockIdx.x * 32 + warp;
    if (lane == 0 && row < rows) {
        // max + log(sum): one rounding of lse, and a loss that is exact to that of log(sum) where
        // the label has the largest logit
        const float rest = R.ctl->failed ? nan_f() : logf(b.y);
        lse[R.index[row]] = R.ctl->failed ? nan_f() : sum ? b.x : b.x + rest;
        if (sum) sum[R.index[row]] = b.y;
        loss[R.index[row]] = b.x - R.picked[row] + rest;
    }
}

// grad_hidden of every row of the call from the sums of its place; a thread takes 4 columns.
template <typename T>
__global__ void __launch_bounds__(256) xent_hidden_kernel(Rows R, const float *sum, T *gh, int64_t M, int64_t Mp,
                                                          int32_t D, int32_t Dq, int32_t splits) {
    pdl_begin();
    const int32_t quads = (D + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, r = i / quads;
    if (r >= M) return;
    const int32_t d = (int32_t)(i % quads) * 4;
    const int at = R.where[r];
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at >= 0) {
        const float *p = sum + (int64_t)at * Dq + d;
        for (int s = 0; s < splits; s += 4) {
            float4 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                q[u] = s + u < splits ? __ldg(reinterpret_cast<const float4 *>(p + (int64_t)(s + u) * Mp * Dq))
                                      : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                v.x += q[u].x;
                v.y += q[u].y;
                v.z += q[u].z;
                v.w += q[u].w;
            }
        }
    }
    if (at == kBadLabel || R.ctl->failed) v = make_float4(nan_f(), nan_f(), nan_f(), nan_f());
    T *to = gh + r * D + d;
    if (D % 4 == 0 && reinterpret_cast<uintptr_t>(gh) % (4 * sizeof(T)) == 0) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(to) = v;
        } else {
            *reinterpret_cast<uint2 *>(to) = make_uint2(two(__float2bfloat16_rn(v.x), __float2bfloat16_rn(v.y)),
                                                        two(__float2bfloat16_rn(v.z), __float2bfloat16_rn(v.w)));
        }
    } else {
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) to[j] = from_f<T>(e[j]);
    }
}

// ------------------------------------------------------------------ host
constexpr size_t kPieceBytes = size_t(512) << 20;   // of G, but at least
constexpr int kLeastTiles = 16;                     // tiles of columns: shorter sums would be bound by joining them
constexpr int kClusters = 76;                        // pairs of the card's 152 SMs

struct Plan {
    int terms;                      // of the operands
    int gterms;                     // of G
    int64_t Mp;                     // rows, a multiple of the tile
    int32_t Dp, Dq;                 // packed row, row of the sums
    int32_t nt, dt, mt;             // tiles along the vocabulary, D and the rows
    int32_t pitch;                  // columns of a piece
    int32_t splits, kb_split;       // of the sum over a piece in HIDDEN
    bool few;                       // the forward takes the float32 operands as they are
    int32_t parts;                  // partial maxima and sums of a row
    // offsets in the scratch buffer
    size_t index, label, where, lse, scale, weight, picked, part, H, W, G, sum;
    size_t bytes;                   // of the scratch buffer, for the pass that was asked for
};

int32_t up(int64_t v, int64_t to) { return (int32_t)((v + to - 1) / to * to); }

// How the backward is cut: into pieces of the vocabulary (G of one within kPieceBytes) and the
// sum over a piece of HIDDEN into splits. The time of a product is that of its fullest pair of
// blocks, so both are chosen by what the card's kClusters pairs take in all, in units of one
// block of kTileK of a tile (0.27 us): 256 tiles of HIDDEN (8192 rows of
// 2048) are 4 rounds of 76 unsplit, and 7 half rounds in two splits.
void choose_pieces(Plan *pl) {
    Plan &p = *pl;
    const int64_t row = std::max<int64_t>(p.Mp, 1) * p.gterms * 2, most = std::max<int64_t>(kLeastTiles, (int64_t)kPieceBytes / (row * kTileN));
    const int32_t fewest = (int32_t)((p.nt + most - 1) / most), kd = p.Dp / kTileK, km = (int32_t)(p.Mp / kTileK);
    const int64_t mt = std::max(p.mt, 1);
    const int times = p.terms == 1 ? p.gterms : 1;   // products of terms in HIDDEN and WEIGHT for one in PIECE
    auto rounds = [](int64_t tiles) { return (tiles + kClusters - 1) / kClusters; };
    double best = 1e300;
    for (int32_t n = fewest; n < fewest + 6 && n <= p.nt; ++n) {
        const int32_t vt = (p.nt + n - 1) / n, kv = vt * (kTileN / kTileK), pieces = (p.nt + vt - 1) / vt;
        for (int32_t s = 1; s <= 32; ++s) {
            const int32_t split = (kv + s - 1) / s;
            if (s > 1 && split < 8) break;
            const double join = (double)s * p.Mp * p.Dq * 8 / 1.6e6;   // bytes of the sums, read and written
            const double cost = pieces * (rounds(mt * vt) * kd + times * (rounds(mt * p.dt * s) * split + rounds((int64_t)vt * p.dt) * km) +
                                          join + 45.0);                // and three launches
            if (cost < best) {
                best = cost;
                p.pitch = vt * kTileN;
                p.kb_split = split;
                p.splits = (kv + split - 1) / split;
            }
        }
    }
}

dendsn_status make_plan(const dendsn_xent_config *cfg, bool backward, Plan *pl) {
    *pl = Plan{};
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->M < 0 || cfg->V < 1 || cfg->D < 1)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad size (M=%d V=%d D=%d)", cfg->M, cfg->V, cfg->D);
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad x_dtype %d", cfg->x_dtype);
    if (cfg->labels_dtype != DENDSN_I32 && cfg->labels_dtype != DENDSN_I64)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad labels_dtype %d", cfg->labels_dtype);
    if (cfg->logit_grad != DENDSN_LOGIT_GRAD_SPLIT && cfg->logit_grad != DENDSN_LOGIT_GRAD_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad logit_grad %d", cfg->logit_grad);
    if (cfg->logit_grad == DENDSN_LOGIT_GRAD_BF16 && cfg->x_dtype == DENDSN_F32)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "a bfloat16 logit_grad is for bfloat16 operands");
    if (cfg->weight_aligned & ~1) return seq_fail(DENDSN_ERR_INVALID_ARG, "weight_aligned must be 0 or 1");
    if (cfg->statistics != DENDSN_STATISTICS_LSE && cfg->statistics != DENDSN_STATISTICS_MAX_SUM)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad statistics %d", cfg->statistics);
    if (cfg->M > (1 << 30) || cfg->V > (1 << 30) || cfg->D > (1 << 24))
        return seq_fail(DENDSN_ERR_UNSUPPORTED, "size out of range (M=%d V=%d D=%d)", cfg->M, cfg->V, cfg->D);
    Plan &p = *pl;
    p.terms = cfg->x_dtype == DENDSN_F32 ? 3 : 1;
    p.gterms = cfg->x_dtype == DENDSN_F32 ? 3 : cfg->logit_grad == DENDSN_LOGIT_GRAD_BF16 ? 1 : 2;
    p.Mp = up(cfg->M, kTileM);
    p.Dp = up(cfg->D, kTileK);
    p.Dq = up(cfg->D, kTileN);
    p.mt = (int32_t)(p.Mp / kTileM);
    p.nt = up(cfg->V, kTileN) / kTileN;
    p.dt = p.Dq / kTileN;
    if (backward) choose_pieces(&p);
    size_t at = sizeof(Ctl);
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    p.index = take(p.Mp * 4);
    p.label = take(p.Mp * 4);
    p.where = take((size_t)cfg->M * 4);
    // statistics for a backward are those of the logits that it will form
    p.few = cfg->x_dtype == DENDSN_F32 && cfg->M <= kFewF32 && cfg->statistics == DENDSN_STATISTICS_LSE;
    const bool packed = backward || !p.few;
    p.H = take(packed ? (size_t)p.terms * p.Mp * p.Dp * 2 : 0);
    // weights are packed unless their rows can be copied as they are, which also their address
    // decides: the caller may say that it is aligned
    const bool as_they_are = cfg->x_dtype == DENDSN_BF16 && cfg->D % 8 == 0 && cfg->weight_aligned;
    p.W = take(packed && !as_they_are ? (size_t)p.terms * cfg->V * p.Dp * 2 : 0);
    if (!backward) {
        p.picked = take(p.Mp * 4);
        p.parts = p.few ? up(cfg->V, kFewV) / kFewV : 2 * p.nt;
        p.part = take((size_t)p.parts * p.Mp * 8);
        p.bytes = at;
        return DENDSN_OK;
    }
    p.lse = take(p.Mp * 4);
    p.scale = take(p.Mp * 4);
    p.weight = take(p.Mp * 4);
    p.G = take((size_t)p.gterms * p.Mp * p.pitch * 2);
    p.sum = take((size_t)p.splits * p.Mp * p.Dq * 4);
    p.bytes = at;
    return DENDSN_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static std::mutex mutex;
    static EncodeTiled fn = nullptr;
    std::lock_guard<std::mutex> lock(mutex);
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult got;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got) == cudaSuccess &&
            got == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiled>(p);
    }
    return fn;
}

// A [planes][rows][inner] bfloat16 tensor read in boxes of 64 x box_rows, zeros outside.
bool make_map(CUtensorMap *map, const void *base, int64_t inner, int64_t rows, int64_t pitch, int planes,
              int64_t plane, int box_rows) {
    EncodeTiled fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)plane * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, ones,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, typename T>
cudaError_t product(const CUtensorMap &a, const CUtensorMap &b, const Gemm &g, int64_t items, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(xent_product_kernel<MODE, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)kSmem);
    if (e != cudaSuccess) return e;
    const unsigned clusters = (unsigned)std::max<int64_t>(1, std::min<int64_t>(items, kClusters));
    return seq_launch(xent_product_kernel<MODE, T>, dim3(2 * clusters), kThreads, kSmem, s, 1, a, b, g);
}

struct Call {
    const dendsn_xent_config *cfg;
    Plan pl;
    char *scratch;
    cudaStream_t s;
    int launches;
    template <typename P> P *at(size_t offset) const { return reinterpret_cast<P *>(scratch + offset); }
};

Rows rows_of(const Call &c) {
    Rows r{};
    r.ctl = c.at<Ctl>(0);
    r.index = c.at<int32_t>(c.pl.index);
    r.label = c.at<int32_t>(c.pl.label);
    r.where = c.at<int32_t>(c.pl.where);
    r.lse = c.at<float>(c.pl.lse);
    r.scale = c.at<float>(c.pl.scale);
    r.weight = c.at<float>(c.pl.weight);
    r.picked = c.at<float>(c.pl.picked);
    return r;
}

// The operands both passes share: the rows that take part, packed, and the weights packed or as
// they are.
template <typename T, typename I>
cudaError_t operands(Call &c, const void *hidden, const void *weight, const PerRow &r, const __nv_bfloat16 **w,
                     int32_t *w_pitch, int64_t *w_inner) {
    const Plan &p = c.pl;
    const int D = c.cfg->D, M = c.cfg->M, V = c.cfg->V;
    const int64_t ignore = c.cfg->ignore_index;
    auto is_wide = [&](const void *from) { return D * sizeof(T) % 16 == 0 && seq_aligned(from, 16); };
    auto pack = [&](const void *from, size_t to, const int32_t *index, int64_t rows) {
        const auto kernel = is_wide(from) ? xent_pack_kernel<T, true> : xent_pack_kernel<T, false>;
        c.launches += 1;
        return seq_launch(kernel, dim3((unsigned)((rows + 7) / 8)), 256, 0, c.s, 1, static_cast<const T *>(from),
                          c.at<__nv_bfloat16>(to), index, c.at<Ctl>(0), rows, D, p.Dp, rows * p.Dp);
    };
    cudaError_t e;
    c.launches += 1;
    if (M <= kFewRows) {
        const auto kernel = is_wide(hidden) ? xent_rows_pack_kernel<T, I, true> : xent_rows_pack_kernel<T, I, false>;
        e = seq_launch(kernel, dim3((unsigned)(p.Mp / 8)), 256, 0, c.s, 1, rows_of(c), r, M, V, ignore, static_cast<const T *>(hidden), c.at<__nv_bfloat16>(p.H), D, p.Dp, p.Mp * p.Dp);
    } else {
        e = seq_launch(xent_rows_kernel<I>, dim3(1), 1024, 0, c.s, 1, rows_of(c), r, M, V, ignore);
        if (e == cudaSuccess) e = pack(hidden, p.H, c.at<int32_t>(p.index), p.Mp);
    }
    if (sizeof(T) == 2 && D % 8 == 0 && seq_aligned(weight, 16)) {
        *w = static_cast<const __nv_bfloat16 *>(weight);
        *w_pitch = D;
        *w_inner = D;
    } else {
        if (e == cudaSuccess) e = pack(weight, p.W, nullptr, V);
        *w = c.at<__nv_bfloat16>(p.W);
        *w_pitch = p.Dp;
        *w_inner = p.Dp;
    }
    return e;
}

template <typename T>
cudaError_t operands(Call &c, const void *hidden, const void *weight, const PerRow &r, const __nv_bfloat16 **w,
                     int32_t *w_pitch, int64_t *w_inner) {
    return c.cfg->labels_dtype == DENDSN_I64 ? operands<T, int64_t>(c, hidden, weight, r, w, w_pitch, w_inner)
                                             : operands<T, int32_t>(c, hidden, weight, r, w, w_pitch, w_inner);
}

// The statistics of few float32 rows.
cudaError_t few_statistics(Call &c, const void *hidden, const void *weight, const PerRow &r) {
    const Plan &p = c.pl;
    const int D = c.cfg->D, M = c.cfg->M, V = c.cfg->V;
    c.launches += 2;
    const auto rows = c.cfg->labels_dtype == DENDSN_I64 ? xent_rows_kernel<int64_t> : xent_rows_kernel<int32_t>;
    cudaError_t e = seq_launch(rows, dim3(1), 1024, 0, c.s, 1, rows_of(c), r, M, V, c.cfg->ignore_index);
    if (e != cudaSuccess) return e;
    const bool wide = D % 4 == 0 && seq_aligned(hidden, 16) && seq_aligned(weight, 16), small = M <= 16;
    const auto kernel = small ? (wide ? xent_few_kernel<16, true> : xent_few_kernel<16, false>)
                              : (wide ? xent_few_kernel<32, true> : xent_few_kernel<32, false>);
    const size_t smem = small ? kFewSmem<16> : kFewSmem<32>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return seq_launch(kernel, dim3((unsigned)p.parts), 256, smem, c.s, 1, rows_of(c), static_cast<const float *>(hidden),
                      static_cast<const float *>(weight), c.at<float2>(p.part), V, D, p.Mp);
}

template <typename T>
dendsn_status run_forward(Call &c, const void *hidden, const void *weight, const void *labels, float *loss, float *lse) {
    const Plan &p = c.pl;
    const int V = c.cfg->V;
    const __nv_bfloat16 *w = nullptr;
    int32_t w_pitch = 0;
    int64_t w_inner = 0;
    cudaError_t e;
    float *sum = c.cfg->statistics == DENDSN_STATISTICS_MAX_SUM ? lse + c.cfg->M : nullptr;
    const PerRow r{labels, loss, lse, sum, nullptr, nullptr, nullptr};
    if (p.few) {
        e = few_statistics(c, hidden, weight, r);
    } else {
        e = operands<T>(c, hidden, weight, r, &w, &w_pitch, &w_inner);
    }
    CUtensorMap a, b;
    if (e == cudaSuccess && !p.few) {
        if (!make_map(&a, c.at<void>(p.H), p.Dp, p.Mp, p.Dp, p.terms, p.Mp * p.Dp, 128) ||
            !make_map(&b, w, w_inner, V, w_pitch, p.terms, (int64_t)V * w_pitch, 128))
            return seq_fail(DENDSN_ERR_CUDA, "tensor map refused");
        Gemm g{};
        g.ctl = c.at<Ctl>(0);
        g.label = c.at<int32_t>(p.label);
        g.picked = c.at<float>(p.picked);
        g.part = c.at<float2>(p.part);
        g.Mp = p.Mp;
        g.nt = p.nt;
        g.splits = 1;
        g.kb = g.kb_split = p.Dp / kTileK;
        g.V = V;
        g.D = c.cfg->D;
        e = product<STATS, T>(a, b, g, (int64_t)p.mt * p.nt, c.s);
        c.launches += 1;
    }
    if (e == cudaSuccess) {
        e = seq_launch(xent_join_kernel, dim3((unsigned)((p.Mp + 31) / 32)), 1024, 0, c.s, 1, rows_of(c), c.at<float2>(p.part),
                       p.parts, p.Mp, loss, lse, sum);
        c.launches += 1;
    }
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "xent forward launch failed: %s", cudaGetErrorString(e));
    return DENDSN_OK;
}

template <typename T>
dendsn_status run_backward(Call &c, const void *hidden, const void *weight, const void *labels, const float *lse,
                           const float *gloss, void *gh, void *gw) {
    const Plan &p = c.pl;
    const int V = c.cfg->V, D = c.cfg->D;
    const __nv_bfloat16 *w = nullptr;
    int32_t w_pitch = 0;
    int64_t w_inner = 0;
    const float *sums = c.cfg->statistics == DENDSN_STATISTICS_MAX_SUM ? lse + c.cfg->M : nullptr;
    cudaError_t e = operands<T>(c, hidden, weight, PerRow{labels, nullptr, nullptr, nullptr, lse, sums, gloss}, &w, &w_pitch, &w_inner);
    CUtensorMap h_rows, h_cols, w_rows, w_cols;
    const __nv_bfloat16 *H = c.at<__nv_bfloat16>(p.H);
    __nv_bfloat16 *G = c.at<__nv_bfloat16>(p.G);
    const int64_t hplane = p.Mp * p.Dp, wplane = (int64_t)V * w_pitch, gplane = p.Mp * p.pitch;
    if (e == cudaSuccess &&
        (!make_map(&h_rows, H, p.Dp, p.Mp, p.Dp, p.terms, hplane, 128) ||
         !make_map(&h_cols, H, p.Dp, p.Mp, p.Dp, p.terms, hplane, 64) ||
         !make_map(&w_rows, w, w_inner, V, w_pitch, p.terms, wplane, 128) ||
         !make_map(&w_cols, w, w_inner, V, w_pitch, p.terms, wplane, 64)))
        return seq_fail(DENDSN_ERR_CUDA, "tensor map refused");
    Gemm g{};
    g.ctl = c.at<Ctl>(0);
    g.label = c.at<int32_t>(p.label);
    g.lse = c.at<float>(p.lse);
    g.scale = c.at<float>(p.scale);
    g.weight = c.at<float>(p.weight);
    g.G = G;
    g.sum = c.at<float>(p.sum);
    g.gw = gw;
    g.Mp = p.Mp;
    g.gplane = gplane;
    g.gterms = p.gterms;
    g.pitch = p.pitch;
    g.V = V;
    g.D = D;
    g.wide = D * sizeof(T) % 32 == 0 && seq_aligned(gw, 32);
    for (int32_t v0 = 0; e == cudaSuccess && v0 < V; v0 += p.pitch) {
        g.v0 = v0;
        g.vc = std::min(p.pitch, V - v0);
        CUtensorMap g_rows, g_cols;
        if (!make_map(&g_rows, G, g.vc, p.Mp, p.pitch, p.gterms, gplane, 128) ||
            !make_map(&g_cols, G, g.vc, p.Mp, p.pitch, p.gterms, gplane, 64))
            return seq_fail(DENDSN_ERR_CUDA, "tensor map refused");
        const int32_t vt = up(g.vc, kTileM) / kTileM;
        g.nt = vt;
        g.splits = 1;
        g.kb = g.kb_split = p.Dp / kTileK;
        e = product<PIECE, T>(h_rows, w_rows, g, (int64_t)p.mt * vt, c.s);
        if (e != cudaSuccess) break;
        g.nt = p.dt;
        g.splits = p.splits;
        g.kb = up(g.vc, kTileK) / kTileK;
        g.kb_split = p.kb_split;
        e = product<HIDDEN, T>(g_rows, w_cols, g, (int64_t)p.mt * p.dt * p.splits, c.s);
        if (e != cudaSuccess) break;
        g.mt = vt;
        g.nt = p.dt;
        g.splits = 1;
        e = product<WEIGHT, T>(g_cols, h_cols, g, (int64_t)vt * p.dt, c.s);
        c.launches += 3;
    }
    if (e == cudaSuccess) {
        const int64_t threads = (int64_t)c.cfg->M * ((D + 3) / 4);
        e = seq_launch(xent_hidden_kernel<T>, dim3((unsigned)((threads + 255) / 256)), 256, 0, c.s, 1, rows_of(c),
                       c.at<float>(p.sum), static_cast<T *>(gh), c.cfg->M, p.Mp, D, p.Dq, p.splits);
        c.launches += 1;
    }
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "xent backward launch failed: %s", cudaGetErrorString(e));
    return DENDSN_OK;
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_xent_workspace_size(const dendsn_xent_config *cfg, size_t *forward_bytes,
                                         size_t *backward_bytes) {
    Plan forward, backward;
    dendsn_status st = make_plan(cfg, false, &forward);
    if (st == DENDSN_OK && backward_bytes) st = make_plan(cfg, true, &backward);
    if (st != DENDSN_OK) return st;
    if (forward_bytes) *forward_bytes = forward.bytes;
    if (backward_bytes) *backward_bytes = backward.bytes;
    return DENDSN_OK;
}

dendsn_status dendsn_xent_forward(const dendsn_xent_config *cfg, const void *hidden, const void *weight,
                                  const void *labels, float *loss, float *lse, void *scratch,
                                  void *stream) {
    Call c{};
    dendsn_status st = make_plan(cfg, false, &c.pl);
    if (st != DENDSN_OK) return st;
    if (cfg->M == 0) return DENDSN_OK;
    if (!hidden || !weight || !labels || !loss || !lse)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "hidden, weight, labels, loss or lse is NULL");
    const bool bf = cfg->x_dtype == DENDSN_BF16, i64 = cfg->labels_dtype == DENDSN_I64;
    if (!seq_aligned(hidden, bf ? 2 : 4) || !seq_aligned(weight, bf ? 2 : 4) || !seq_aligned(labels, i64 ? 8 : 4) ||
        !seq_aligned(loss, 4) || !seq_aligned(lse, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "a tensor is misaligned");
    if (cfg->weight_aligned && !seq_aligned(weight, 16))
        return seq_fail(DENDSN_ERR_MISALIGNED, "weight is not 16-byte aligned, as weight_aligned says");
    if (!scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 256-byte aligned");
    c.cfg = cfg;
    c.scratch = static_cast<char *>(scratch);
    c.s = static_cast<cudaStream_t>(stream);
    st = bf ? run_forward<__nv_bfloat16>(c, hidden, weight, labels, loss, lse)
            : run_forward<float>(c, hidden, weight, labels, loss, lse);
    seq_count_launches(c.launches);
    return st;
}

dendsn_status dendsn_xent_backward(const dendsn_xent_config *cfg, const void *hidden, const void *weight,
                                   const void *labels, const float *lse, const float *grad_loss,
                                   void *grad_hidden, void *grad_weight, void *scratch, void *stream) {
    Call c{};
    dendsn_status st = make_plan(cfg, true, &c.pl);
    if (st != DENDSN_OK) return st;
    if (!grad_weight || !weight) return seq_fail(DENDSN_ERR_INVALID_ARG, "weight or grad_weight is NULL");
    if (cfg->M > 0 && (!hidden || !labels || !lse || !grad_loss || !grad_hidden))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "hidden, labels, lse, grad_loss or grad_hidden is NULL");
    const bool bf = cfg->x_dtype == DENDSN_BF16, i64 = cfg->labels_dtype == DENDSN_I64;
    const size_t sx = bf ? 2 : 4;
    if (!seq_aligned(hidden, sx) || !seq_aligned(weight, sx) || !seq_aligned(grad_hidden, sx) ||
        !seq_aligned(grad_weight, sx) || !seq_aligned(labels, i64 ? 8 : 4) || !seq_aligned(lse, 4) ||
        !seq_aligned(grad_loss, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "a tensor is misaligned");
    if (cfg->weight_aligned && !seq_aligned(weight, 16))
        return seq_fail(DENDSN_ERR_MISALIGNED, "weight is not 16-byte aligned, as weight_aligned says");
    if (!scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 256-byte aligned");
    c.cfg = cfg;
    c.scratch = static_cast<char *>(scratch);
    c.s = static_cast<cudaStream_t>(stream);
    if (cfg->M == 0) {
        cudaError_t e = cudaMemsetAsync(grad_weight, 0, (size_t)cfg->V * cfg->D * sx, c.s);
        if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "memset failed: %s", cudaGetErrorString(e));
        return DENDSN_OK;
    }
    st = bf ? run_backward<__nv_bfloat16>(c, hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight)
            : run_backward<float>(c, hidden, weight, labels, lse, grad_loss, grad_hidden, grad_weight);
    seq_count_launches(c.launches);
    return st;
}

}  // extern "C"
