// Root-mean-square norm with the residual's addition, and its gradient:
//   z = round(x + residual),  r = 1 / sqrt(mean(z^2) + eps),  y = z r w
//   h = g w,  grad_x = r (h - z r^2 mean(h z)) + grad_sum,  grad_w = sum over rows of g z r
// y goes out in the inputs' type, or as e4m3 codes with a float32 scale for a row or for each 128
// columns (the largest of a group becomes 448).
//
// Both are bound by memory: a row is read once into registers, its statistics are formed there and
// it is written from there. A row of up to 32 values a lane is one warp's (sums by shuffles alone);
// a longer one is a block's, of as few warps as hold it. The backward forms r again from z instead
// of reading it. Its column sums stay in each thread's registers over all rows of a block and go to
// a [blocks, D] table, which a second launch adds up in order: no atomics, the same sums from run to
// run.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "pieces.cuh"
#include "seq_common.h"

namespace dendsn {
namespace {

constexpr int kMostColumns = 16384;
constexpr int kWarpRows = 4;          // rows of a block whose rows have a warp each
constexpr int kGroup = 128;           // columns that share a scale
constexpr int kBlocks = 152 * 4;      // of the backward at most: rows of the table of column sums
constexpr int kSumColumns = 8, kSumRows = 64;

// Where vector j of a thread lies in its row. Vectors of 16 bytes are dealt out lane by lane;
// single elements in runs of 128, so that the columns of a scale belong to one warp.
template <int VEC>
__device__ __forceinline__ int place(int j, int thread, int threads) {
    if (VEC > 1) return j * threads + thread;
    return ((j >> 2) * (threads >> 5) + (thread >> 5)) * 128 + (j & 3) * 32 + (thread & 31);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v, int from) {
    for (int o = from; o; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// Two sums over the threads of a row. `red` alternates between calls, so one barrier a call is enough.
__device__ __forceinline__ float2 row_sums(float a, float b, int threads, float2 *red) {
    a = warp_sum(a);
    b = warp_sum(b);
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
        for (int w = 0; w < threads >> 5; ++w) a += red[w].x, b += red[w].y;
    }
    return make_float2(a, b);
}

template <int VEC>
__device__ __forceinline__ void weights(float (&w)[VEC], const float *weight, int k) {
    if (VEC == 1) {
        w[0] = __ldg(weight + k);
    } else {
#pragma unroll
        for (int e = 0; e < VEC / 4; ++e) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(weight + k * VEC) + e);
            w[4 * e] = q.x, w[4 * e + 1] = q.y, w[4 * e + 2] = q.z, w[4 * e + 3] = q.w;
        }
    }
}

// Sizes as unsigned integers order as the sizes do, and a NaN is above them all.
__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// The scale that makes the largest of a group 448, and its reciprocal. A group whose
// largest is below 2^-100 (none of a model's) keeps scale 1, where its codes are zeros.
__device__ __forceinline__ float2 scale_of(uint32_t top) {
    const float t = __uint_as_float(top);
    if (t < 0x1p-100f) return make_float2(1.f, 1.f);
    const float s = t * (1.f / 448.f);
    return make_float2(s, __frcp_rn(s));
}
// v / scale as the division rounds it (the approximate quotient corrected by what it leaves, Markstein's division step): a
// code is decided by the quotient's last bits only.
__device__ __forceinline__ float scaled(float v, float2 s) {
    const float q = v * s.y;
    return fmaf(fmaf(-q, s.x, v), s.y, q);
}

struct Rows {
    int64_t M;
    int32_t D, nv;             // columns, vectors of a row
    int32_t threads;           // of a row
    float eps;
};

// OUT: 0 the inputs' type, 1 e4m3 with a scale for a row, 2 e4m3 with a scale for 128 columns.
template <typename T, int VEC, int NV, int OUT>
__global__ void __launch_bounds__(512) norm_forward_kernel(const T *x, const T *residual, const float *weight, T *sum,
                                                           void *y, float *scales, Rows p) {
    using L = Lot<T, VEC>;
    __shared__ float2 red[2][16];
    __shared__ uint32_t tops[16];
    pdl_begin();
    const int rows = blockDim.x / p.threads, thread = threadIdx.x % p.threads;
    const int groups = (p.D + kGroup - 1) / kGroup;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / p.threads; row < p.M; row += (int64_t)gridDim.x * rows, turn ^= 1) {
        const L *xr = reinterpret_cast<const L *>(x) + row * p.nv;
        L z[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = place<VEC>(j, thread, p.threads);
            z[j].zero();
            if (k < p.nv) z[j] = xr[k];
        }
        if (residual) {
            const L *rr = reinterpret_cast<const L *>(residual) + row * p.nv;
            L *sr = reinterpret_cast<L *>(sum) + row * p.nv;
            L q[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = place<VEC>(j, thread, p.threads);
                q[j].zero();
                if (k < p.nv) q[j] = rr[k];
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = place<VEC>(j, thread, p.threads);
                float a[VEC], b[VEC];
                z[j].get(a);
                q[j].get(b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) a[e] += b[e];
                z[j].set(a);
                if (k < p.nv) sr[k] = z[j];
            }
        }
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float v[VEC];
            z[j].get(v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) ss = fmaf(v[e], v[e], ss);
        }
        ss = row_sums(ss, 0.f, p.threads, red[turn]).x;
        const float r = __fdiv_rn(1.f, sqrtf(ss / (float)p.D + p.eps));
        uint32_t top = 0;
        float2 scale[OUT == 2 && VEC == 1 ? (NV + 3) / 4 : 1];
        if (OUT == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = place<VEC>(j, thread, p.threads);
                float v[VEC], w[VEC];
                z[j].get(v);
                if (k < p.nv) {
                    weights<VEC>(w, weight, k);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) top = max(top, size_bits(v[e] * r * w[e]));
                }
            }
            top = warp_max(top, 16);
            if (p.threads > 32) {
                if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
                __syncthreads();       // the next row's sums stand between this read and the next write
                top = 0;
                for (int w = 0; w < p.threads >> 5; ++w) top = max(top, tops[w]);
            }
            const float2 s = scale_of(top);
            scale[0] = s;
            if (thread == 0) scales[row] = s.x;
        }
        if (OUT == 2 && VEC == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int k = place<VEC>(j, thread, p.threads);
                float v[VEC];
                z[j].get(v);
                if (j % 4 == 0) top = 0;
                if (k < p.nv) top = max(top, size_bits(v[0] * r * __ldg(weight + k)));
                if (j % 4 == 3) {
                    const float2 s = scale_of(warp_max(top, 16));
                    scale[j / 4] = s;
                    const int first = k - (k & 127);
                    if ((thread & 31) == 0 && first < p.D) scales[row * groups + first / kGroup] = s.x;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = place<VEC>(j, thread, p.threads);
            float v[VEC];
            z[j].get(v);
            if (k < p.nv) {
                float w[VEC];
                weights<VEC>(w, weight, k);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] = v[e] * r * w[e];
            }
            if (OUT == 0) {
                L o;
                o.set(v);
                if (k < p.nv) reinterpret_cast<L *>(y)[row * p.nv + k] = o;
                continue;
            }
            float2 by = OUT == 2 && VEC == 1 ? scale[j / 4] : scale[0];
            if (OUT == 2 && VEC > 1) {       // 128 columns are 128 / VEC neighbouring lanes' vector
                top = 0;
                if (k < p.nv)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) top = max(top, size_bits(v[e]));
                const float2 s = scale_of(warp_max(top, 64 / VEC));
                by = s;
                if ((k * VEC) % kGroup == 0 && k < p.nv) scales[row * groups + k * VEC / kGroup] = s.x;
            }
            if (k < p.nv) {
                uint8_t *to = reinterpret_cast<uint8_t *>(y) + row * p.D + k * VEC;
                if (VEC == 1) {
                    *to = (uint8_t)e4m3_pair(scaled(v[0], by), 0.f);
                } else {
                    uint32_t q[VEC / 4 ? VEC / 4 : 1];
#pragma unroll
                    for (int e = 0; e < VEC / 4; ++e)
                        q[e] = (uint32_t)e4m3_pair(scaled(v[4 * e], by), scaled(v[4 * e + 1], by)) |
                               (uint32_t)e4m3_pair(scaled(v[4 * e + 2], by), scaled(v[4 * e + 3], by)) << 16;
                    if (VEC == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(q[0], q[VEC / 4 - 1]);
                    else *reinterpret_cast<uint32_t *>(to) = q[0];
                }
            }
        }
    }
}

// BLOCK: threads it is built for. A block of 128 may have more registers than one of 512.
template <typename T, int VEC, int NV, int BLOCK>
__global__ void __launch_bounds__(BLOCK) norm_backward_kernel(const T *sum, const float *weight, const T *gy,
                                                            const T *gsum, T *gx, float *table, Rows p) {
    using L = Lot<T, VEC>;
    __shared__ float2 red[2][16];
    extern __shared__ float columns[];        // [rows - 1][NV * VEC][32]: where a block's rows have a warp each
    pdl_begin();
    const int rows = blockDim.x / p.threads, thread = threadIdx.x % p.threads, mine = threadIdx.x / p.threads;
    float gw[NV * VEC];
#pragma unroll
    for (int i = 0; i < NV * VEC; ++i) gw[i] = 0.f;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * rows + mine; row < p.M; row += (int64_t)gridDim.x * rows, turn ^= 1) {
        const L *zr = reinterpret_cast<const L *>(sum) + row * p.nv, *gr = reinterpret_cast<const L *>(gy) + row * p.nv;
        const L *ar = reinterpret_cast<const L *>(gsum) + row * p.nv;
        L z[NV], g[NV], q[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = place<VEC>(j, thread, p.threads);
            z[j].zero();
            g[j].zero();
            q[j].zero();
            if (k < p.nv) z[j] = zr[k], g[j] = gr[k];
            if (k < p.nv && gsum) q[j] = ar[k];
        }
        float ss = 0.f, hz = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = place<VEC>(j, thread, p.threads);
            float v[VEC], h[VEC];
            z[j].get(v);
            g[j].get(h);
            if (k < p.nv) {
                float w[VEC];
                weights<VEC>(w, weight, k);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    ss = fmaf(v[e], v[e], ss);
                    hz = fmaf(h[e] * w[e], v[e], hz);
                }
            }
        }
        const float2 s = row_sums(ss, hz, p.threads, red[turn]);
        const float r = __fdiv_rn(1.f, sqrtf(s.x / (float)p.D + p.eps));
        const float along = r * r * (s.y / (float)p.D);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = place<VEC>(j, thread, p.threads);
            float v[VEC], h[VEC], a[VEC];
            z[j].get(v);
            g[j].get(h);
            q[j].get(a);
            if (k < p.nv) {
                float w[VEC];
                weights<VEC>(w, weight, k);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    gw[j * VEC + e] = fmaf(h[e], v[e] * r, gw[j * VEC + e]);
                    a[e] = fmaf(r, fmaf(-along, v[e], h[e] * w[e]), a[e]);
                }
                L o;
                o.set(a);
                (reinterpret_cast<L *>(gx) + row * p.nv)[k] = o;
            }
        }
    }
    if (rows > 1) {
        if (mine)
#pragma unroll
            for (int i = 0; i < NV * VEC; ++i) columns[((mine - 1) * NV * VEC + i) * 32 + thread] = gw[i];
        __syncthreads();
        if (mine) return;
#pragma unroll
        for (int i = 0; i < NV * VEC; ++i)
            for (int w = 1; w < rows; ++w) gw[i] += columns[((w - 1) * NV * VEC + i) * 32 + thread];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int k = place<VEC>(j, thread, p.threads);
        if (k < p.nv)
#pragma unroll
            for (int e = 0; e < VEC; ++e) table[(int64_t)blockIdx.x * p.D + k * VEC + e] = gw[j * VEC + e];
    }
}

// The table's columns added up: 8 columns (a sector) a block, every 64th row by each of a column's threads, in
// order. 16384 rows, D = 1024: 32 columns and 16 threads 8 us.
__global__ void __launch_bounds__(kSumColumns *kSumRows) norm_columns_kernel(const float *table, float *gweight, int32_t blocks, int32_t D) {
    __shared__ float part[kSumRows][kSumColumns];
    pdl_begin();
    const int c = threadIdx.x % kSumColumns, t = threadIdx.x / kSumColumns, col = blockIdx.x * kSumColumns + c;
    float v = 0.f;
    if (col < D) {
#pragma unroll 10
        for (int b = t; b < blocks; b += kSumRows) v += table[(int64_t)b * D + col];
    }
    part[t][c] = v;
    __syncthreads();
    if (t || col >= D) return;
    v = 0.f;
    for (int i = 0; i < kSumRows; ++i) v += part[i][c];
    gweight[col] = v;
}

template <int N> struct Int { static constexpr int value = N; };

struct Plan {
    Rows rows;
    int block, blocks;         // threads of a block, blocks of the grid
    int vectors;               // NV
};

dendsn_status check(const dendsn_norm_config *cfg) {
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->M < 0 || cfg->D < 1) return seq_fail(DENDSN_ERR_INVALID_ARG, "M must be >= 0 and D >= 1");
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown x_dtype");
    if (cfg->out != DENDSN_NORM_SAME && cfg->out != DENDSN_NORM_E4M3) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown out");
    if (cfg->group != 0 && cfg->group != kGroup) return seq_fail(DENDSN_ERR_INVALID_ARG, "group must be 0 (a row) or %d columns", kGroup);
    if (!(cfg->eps >= 0.f) || std::isinf(cfg->eps)) return seq_fail(DENDSN_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (cfg->D > kMostColumns) return seq_fail(DENDSN_ERR_UNSUPPORTED, "rows of more than %d columns", kMostColumns);
    return DENDSN_OK;
}

int blocks_of(const dendsn_norm_config &c, int rows, int most) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(((int64_t)c.M + rows - 1) / rows, most));
}

// Vectors: up to 32 values a thread, a warp for a row where that holds it, four such rows a block. Single
// elements: 8 a thread while a block's 512 threads hold the row so, as each load moves little (1009 rows of
// 1001 floats, backward: 32 a thread 32 us).
Plan plan_of(const dendsn_norm_config &c, bool wide) {
    Plan p;
    const int vec = !wide ? 1 : c.x_dtype == DENDSN_BF16 ? 8 : 4;
    p.rows = {c.M, c.D, c.D / vec, 32, c.eps};
    const int nv = (p.rows.nv + 31) / 32, most = vec > 1 ? 32 / vec : nv <= 8 * 16 ? 8 : nv <= 16 * 16 ? 16 : 32;
    p.vectors = vec == 1 ? 4 : 1;
    while (p.vectors < most && p.vectors < nv) p.vectors *= 2;
    if (nv > p.vectors) p.rows.threads = (nv + p.vectors - 1) / p.vectors * 32;
    p.block = p.rows.threads == 32 ? 32 * kWarpRows : p.rows.threads;
    return p;
}

template <typename T, int VEC, int OUT>
cudaError_t forward_of(const Plan &p, const void *x, const void *res, const float *w, void *sum, void *y, float *scales, cudaStream_t s) {
    auto go = [&](auto kernel) {
        return seq_launch(kernel, dim3((unsigned)p.blocks), p.block, 0, s, 1, (const T *)x, (const T *)res, w, (T *)sum, y, scales, p.rows);
    };
    switch (p.vectors) {
        case 1: return go(norm_forward_kernel<T, VEC, VEC == 1 ? 4 : 1, OUT>);
        case 2: return go(norm_forward_kernel<T, VEC, VEC == 1 ? 4 : 2, OUT>);
        case 4: return go(norm_forward_kernel<T, VEC, 4, OUT>);
        case 8: return go(norm_forward_kernel<T, VEC, VEC == 8 ? 4 : 8, OUT>);
        case 16: return go(norm_forward_kernel<T, VEC, VEC == 1 ? 16 : 4, OUT>);
        default: return go(norm_forward_kernel<T, VEC, VEC == 1 ? 32 : 4, OUT>);
    }
}
template <typename T, int VEC>
cudaError_t forward_out(const dendsn_norm_config &c, const Plan &p, const void *x, const void *res, const float *w, void *sum, void *y, float *scales, cudaStream_t s) {
    if (c.out == DENDSN_NORM_SAME) return forward_of<T, VEC, 0>(p, x, res, w, sum, y, scales, s);
    return c.group ? forward_of<T, VEC, 2>(p, x, res, w, sum, y, scales, s) : forward_of<T, VEC, 1>(p, x, res, w, sum, y, scales, s);
}
template <typename T, int VEC>
cudaError_t backward_of(const Plan &p, const void *sum, const float *w, const void *gy, const void *gsum, void *gx, float *table, cudaStream_t s) {
    auto go = [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        const size_t smem = p.rows.threads == 32 ? (size_t)(kWarpRows - 1) * NV * VEC * 32 * 4 : 0;
        auto run = [&](auto kernel) {
            return seq_launch(kernel, dim3((unsigned)p.blocks), p.block, smem, s, 1, (const T *)sum, w, (const T *)gy, (const T *)gsum, (T *)gx, table, p.rows);
        };
        return p.block <= 128 ? run(norm_backward_kernel<T, VEC, NV, 128>) : run(norm_backward_kernel<T, VEC, NV, 512>);
    };
    switch (p.vectors) {
        case 1: return go(Int<VEC == 1 ? 4 : 1>());
        case 2: return go(Int<VEC == 1 ? 4 : 2>());
        case 4: return go(Int<4>());
        case 8: return go(Int<VEC == 8 ? 4 : 8>());
        case 16: return go(Int<VEC == 1 ? 16 : 4>());
        default: return go(Int<VEC == 1 ? 32 : 4>());
    }
}

// 16-byte vectors: every row of every tensor starts at a multiple of 16 bytes.
bool wide_rows(const dendsn_norm_config &c, std::initializer_list<const void *> tensors, const float *weight) {
    if (c.D % (c.x_dtype == DENDSN_BF16 ? 8 : 4) || !seq_aligned(weight, 16)) return false;
    for (const void *t : tensors)
        if (!seq_aligned(t, 16)) return false;
    return true;
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_norm_workspace_size(const dendsn_norm_config *cfg, size_t *scratch_bytes) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    if (scratch_bytes) *scratch_bytes = (size_t)blocks_of(*cfg, 1, kBlocks) * (size_t)cfg->D * 4;
    return DENDSN_OK;
}

dendsn_status dendsn_norm_forward(const dendsn_norm_config *cfg, const void *x, const void *residual, const float *weight,
                                  void *sum, void *y, float *scales, void *stream) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK || cfg->M == 0) return st;
    const bool eight = cfg->out == DENDSN_NORM_E4M3;
    if (!x || !weight || !y) return seq_fail(DENDSN_ERR_INVALID_ARG, "x, weight or y is NULL");
    if ((residual == nullptr) != (sum == nullptr)) return seq_fail(DENDSN_ERR_INVALID_ARG, "residual and sum go together");
    if (eight && !scales) return seq_fail(DENDSN_ERR_INVALID_ARG, "scales is NULL");
    const size_t sx = cfg->x_dtype == DENDSN_BF16 ? 2 : 4;
    if (!seq_aligned(x, sx) || !seq_aligned(residual, sx) || !seq_aligned(sum, sx) || !seq_aligned(weight, 4) ||
        !seq_aligned(y, eight ? 1 : sx) || !seq_aligned(scales, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "x, residual, weight, sum, y or scales misaligned");
    const bool wide = wide_rows(*cfg, {x, residual, sum}, weight) && seq_aligned(y, eight ? 16 / sx : 16);
    Plan p = plan_of(*cfg, wide);
    p.blocks = blocks_of(*cfg, p.block / p.rows.threads, 1 << 30);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cfg->x_dtype == DENDSN_BF16
                        ? (wide ? forward_out<__nv_bfloat16, 8>(*cfg, p, x, residual, weight, sum, y, scales, s)
                                : forward_out<__nv_bfloat16, 1>(*cfg, p, x, residual, weight, sum, y, scales, s))
                        : (wide ? forward_out<float, 4>(*cfg, p, x, residual, weight, sum, y, scales, s)
                                : forward_out<float, 1>(*cfg, p, x, residual, weight, sum, y, scales, s));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "norm forward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

dendsn_status dendsn_norm_backward(const dendsn_norm_config *cfg, const void *sum, const float *weight, const void *grad_y,
                                   const void *grad_sum, void *grad_x, float *grad_weight, void *scratch, void *stream) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    if (!weight || !grad_weight) return seq_fail(DENDSN_ERR_INVALID_ARG, "weight or grad_weight is NULL");
    if (cfg->M > 0 && (!sum || !grad_y || !grad_x)) return seq_fail(DENDSN_ERR_INVALID_ARG, "sum, grad_y or grad_x is NULL");
    if (!scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    const size_t sx = cfg->x_dtype == DENDSN_BF16 ? 2 : 4;
    if (!seq_aligned(sum, sx) || !seq_aligned(grad_y, sx) || !seq_aligned(grad_sum, sx) || !seq_aligned(grad_x, sx) ||
        !seq_aligned(weight, 4) || !seq_aligned(grad_weight, 4) || !seq_aligned(scratch, 16))
        return seq_fail(DENDSN_ERR_MISALIGNED, "sum, weight, a gradient or scratch (16 bytes) misaligned");
    const bool wide = wide_rows(*cfg, {sum, grad_y, grad_sum, grad_x}, weight);
    Plan p = plan_of(*cfg, wide);
    p.blocks = blocks_of(*cfg, p.block / p.rows.threads, kBlocks);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float *table = static_cast<float *>(scratch);
    cudaError_t e = cfg->x_dtype == DENDSN_BF16
                        ? (wide ? backward_of<__nv_bfloat16, 8>(p, sum, weight, grad_y, grad_sum, grad_x, table, s)
                                : backward_of<__nv_bfloat16, 1>(p, sum, weight, grad_y, grad_sum, grad_x, table, s))
                        : (wide ? backward_of<float, 4>(p, sum, weight, grad_y, grad_sum, grad_x, table, s)
                                : backward_of<float, 1>(p, sum, weight, grad_y, grad_sum, grad_x, table, s));
    if (e == cudaSuccess)
        e = seq_launch(norm_columns_kernel, dim3((unsigned)((cfg->D + kSumColumns - 1) / kSumColumns)), kSumColumns * kSumRows, 0, s, 1,
                       (const float *)table, grad_weight, p.blocks, cfg->D);
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "norm backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(2);
    return DENDSN_OK;
}

}  // extern "C"
