// Softmax cross entropy of a linear readout in pieces of the vocabulary, and its gradient.
#include <cuda_bf16.h>

#include <algorithm>

#include "seq_common.h"

namespace dendsn {
namespace {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr int kTile = 64, kK = 16;
constexpr int kIgnored = -1, kBadLabel = -2;

template <typename I>
__device__ __forceinline__ int label_of(const void *labels, int r, int V, int64_t ignore) {
    const int64_t y = static_cast<const I *>(labels)[r];
    return y == ignore ? kIgnored : (y < 0 || y >= V) ? kBadLabel : (int)y;
}

// acc[i][j] += sum_k A(row0 + 4 ty + i, k) B(col0 + 4 tx + j, k) over k in [0, K), with the
// loaders returning 0 outside their matrices; 256 threads, 64 x 64 tile.
template <typename LA, typename LB>
__device__ __forceinline__ void tile_product(float (&acc)[4][4], int64_t K, LA la, LB lb) {
    __shared__ float As[kK][kTile + 1], Bs[kK][kTile + 1];
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int64_t k0 = 0; k0 < K; k0 += kK) {
        __syncthreads();
        for (int e = threadIdx.x; e < kTile * kK; e += 256) {
            As[e % kK][e / kK] = k0 + e % kK < K ? la(e / kK, k0 + e % kK) : 0.f;
            Bs[e % kK][e / kK] = k0 + e % kK < K ? lb(e / kK, k0 + e % kK) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kK; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(As[k][4 * ty + i], Bs[k][4 * tx + j], acc[i][j]);
    }
}

struct Args {
    const void *hidden, *weight, *labels;
    int64_t ignore;
    int32_t M, V, D;
    float *loss, *lse;
    const float *lse_in, *gloss;
    void *gh, *gw;
    float *G, *gh32;
    int32_t v0, vc;
};

template <typename T, typename I>
__global__ void __launch_bounds__(256) xent_forward_kernel(const Args A) {
    __shared__ int lab[kTile];
    __shared__ float picked[kTile];
    const int64_t r0 = (int64_t)blockIdx.x * kTile;
    const T *H = static_cast<const T *>(A.hidden), *W = static_cast<const T *>(A.weight);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    if (threadIdx.x < kTile) {
        lab[threadIdx.x] = r0 + threadIdx.x < A.M ? label_of<I>(A.labels, r0 + threadIdx.x, A.V, A.ignore) : kIgnored;
        picked[threadIdx.x] = 0.f;
    }
    __syncthreads();
    float top[4], sum[4];
    for (int i = 0; i < 4; ++i) { top[i] = -INFINITY; sum[i] = 0.f; }
    for (int v0 = 0; v0 < A.V; v0 += kTile) {
        float acc[4][4] = {};
        tile_product(acc, A.D,
                     [&](int i, int64_t k) { return lab[i] >= 0 ? to_f<T>(H[(r0 + i) * A.D + k]) : 0.f; },
                     [&](int j, int64_t k) { return v0 + j < A.V ? to_f<T>(W[(int64_t)(v0 + j) * A.D + k]) : 0.f; });
        for (int i = 0; i < 4; ++i) {
            float m = top[i];
            for (int j = 0; j < 4; ++j) {
                const int v = v0 + 4 * tx + j;
                if (v < A.V) m = fmaxf(m, acc[i][j]);
                if (v < A.V && v == lab[4 * ty + i]) picked[4 * ty + i] = acc[i][j];
            }
            const float ref = m == -INFINITY ? 0.f : m;
            float s = sum[i] * expf(top[i] - ref);
            for (int j = 0; j < 4; ++j)
                if (v0 + 4 * tx + j < A.V) s += expf(acc[i][j] - ref);
            top[i] = m;
            sum[i] = s;
        }
    }
    __syncthreads();
    for (int i = 0; i < 4; ++i) {
        for (int o = 8; o; o >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, top[i], o), s2 = __shfl_xor_sync(0xffffffffu, sum[i], o);
            const float m = fmaxf(top[i], m2), ref = m == -INFINITY ? 0.f : m;
            sum[i] = sum[i] * expf(top[i] - ref) + s2 * expf(m2 - ref);
            top[i] = m;
        }
        const int r = 4 * ty + i;
        if (tx == 0 && r0 + r < A.M) {
            const float lse = (top[i] == -INFINITY ? 0.f : top[i]) + logf(sum[i]);
            const float nan = __int_as_float(0x7fffffff);
            A.lse[r0 + r] = lab[r] >= 0 ? lse : lab[r] == kIgnored ? 0.f : nan;
            A.loss[r0 + r] = lab[r] >= 0 ? lse - picked[r] : lab[r] == kIgnored ? 0.f : nan;
        }
    }
}

template <typename T, typename I>
__global__ void __launch_bounds__(256) xent_piece_kernel(const Args A) {
    __shared__ int lab[kTile];
    const int64_t r0 = (int64_t)blockIdx.y * kTile, c0 = (int64_t)blockIdx.x * kTile;
    const T *H = static_cast<const T *>(A.hidden), *W = static_cast<const T *>(A.weight) + (int64_t)A.v0 * A.D;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    if (threadIdx.x < kTile)
        lab[threadIdx.x] = r0 + threadIdx.x < A.M ? label_of<I>(A.labels, r0 + threadIdx.x, A.V, A.ignore) : kIgnored;
    __syncthreads();
    float acc[4][4] = {};
    tile_product(acc, A.D,
                 [&](int i, int64_t k) { return lab[i] >= 0 ? to_f<T>(H[(r0 + i) * A.D + k]) : 0.f; },
                 [&](int j, int64_t k) { return c0 + j < A.vc ? to_f<T>(W[(c0 + j) * A.D + k]) : 0.f; });
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + 4 * ty + i;
        const int y = lab[4 * ty + i];
        if (r >= A.M) continue;
        for (int j = 0; j < 4; ++j) {
            const int64_t c = c0 + 4 * tx + j;
            if (c >= A.vc) continue;
            float g = 0.f;
            if (y >= 0) g = A.gloss[r] * (expf(acc[i][j] - A.lse_in[r]) - (y == A.v0 + c ? 1.f : 0.f));
            A.G[r * A.vc + c] = g;
        }
    }
}

// gh32 (+)= G W of the piece; the last piece writes grad_hidden.
template <typename T, typename I>
__global__ void __launch_bounds__(256) xent_grad_hidden_kernel(const Args A) {
    const int64_t r0 = (int64_t)blockIdx.y * kTile, d0 = (int64_t)blockIdx.x * kTile;
    const T *W = static_cast<const T *>(A.weight) + (int64_t)A.v0 * A.D;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    tile_product(acc, A.vc, [&](int i, int64_t k) { return r0 + i < A.M ? A.G[(r0 + i) * A.vc + k] : 0.f; },
                 [&](int j, int64_t k) { return d0 + j < A.D ? to_f<T>(W[k * A.D + d0 + j]) : 0.f; });
    const bool last = A.v0 + A.vc == A.V;
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + 4 * ty + i;
        if (r >= A.M) continue;
        const int y = label_of<I>(A.labels, r, A.V, A.ignore);
        for (int j = 0; j < 4; ++j) {
            const int64_t d = d0 + 4 * tx + j;
            if (d >= A.D) continue;
            float v = acc[i][j] + (A.v0 ? A.gh32[r * A.D + d] : 0.f);
            A.gh32[r * A.D + d] = v;
            if (y < 0) v = y == kIgnored ? 0.f : __int_as_float(0x7fffffff);
            if (last) static_cast<T *>(A.gh)[r * A.D + d] = from_f<T>(v);
        }
    }
}

template <typename T, typename I>
__global__ void __launch_bounds__(256) xent_grad_weight_kernel(const Args A) {
    const int64_t c0 = (int64_t)blockIdx.y * kTile, d0 = (int64_t)blockIdx.x * kTile;
    const T *H = static_cast<const T *>(A.hidden);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    tile_product(acc, A.M, [&](int i, int64_t k) { return c0 + i < A.vc ? A.G[k * A.vc + c0 + i] : 0.f; },
                 [&](int j, int64_t k) {
                     return d0 + j < A.D && label_of<I>(A.labels, k, A.V, A.ignore) >= 0
                                ? to_f<T>(H[k * A.D + d0 + j]) : 0.f;
                 });
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t c = c0 + 4 * ty + i, d = d0 + 4 * tx + j;
            if (c < A.vc && d < A.D) static_cast<T *>(A.gw)[(A.v0 + c) * A.D + d] = from_f<T>(acc[i][j]);
        }
}

constexpr int kPiece = 4096;

struct Plan {
    size_t fwd = 0, bwd = 0, gh32 = 0;
};

dendsn_status make_plan(const dendsn_xent_config *cfg, Plan *pl) {
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->M < 0 || cfg->V < 1 || cfg->D < 1)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad size (M=%d V=%d D=%d)", cfg->M, cfg->V, cfg->D);
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad x_dtype %d", cfg->x_dtype);
    if (cfg->labels_dtype != DENDSN_I32 && cfg->labels_dtype != DENDSN_I64)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad labels_dtype %d", cfg->labels_dtype);
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    pl->gh32 = up((size_t)cfg->M * cfg->D * 4);
    pl->bwd = pl->gh32 + up((size_t)cfg->M * std::min(cfg->V, kPiece) * 4);
    return DENDSN_OK;
}

unsigned tiles(int64_t n) { return (unsigned)((n + kTile - 1) / kTile); }

template <typename T, typename I>
cudaError_t run_forward(const Args &a, cudaStream_t s) {
    xent_forward_kernel<T, I><<<tiles(a.M), 256, 0, s>>>(a);
    return cudaGetLastError();
}

template <typename T, typename I>
cudaError_t run_backward(Args a, cudaStream_t s, int *launches) {
    for (int v0 = 0; v0 < a.V; v0 += kPiece) {
        a.v0 = v0;
        a.vc = std::min(kPiece, a.V - v0);
        if (a.M > 0) {
            xent_piece_kernel<T, I><<<dim3(tiles(a.vc), tiles(a.M)), 256, 0, s>>>(a);
            xent_grad_hidden_kernel<T, I><<<dim3(tiles(a.D), tiles(a.M)), 256, 0, s>>>(a);
            *launches += 2;
        }
        xent_grad_weight_kernel<T, I><<<dim3(tiles(a.D), tiles(a.vc)), 256, 0, s>>>(a);
        *launches += 1;
    }
    return cudaGetLastError();
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_xent_workspace_size(const dendsn_xent_config *cfg, size_t *forward_bytes,
                                         size_t *backward_bytes) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
    if (st != DENDSN_OK) return st;
    if (forward_bytes) *forward_bytes = pl.fwd;
    if (backward_bytes) *backward_bytes = pl.bwd;
    return DENDSN_OK;
}

dendsn_status dendsn_xent_forward(const dendsn_xent_config *cfg, const void *hidden, const void *weight,
                                  const void *labels, float *loss, float *lse, void *scratch,
                                  void *stream) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
    if (st != DENDSN_OK) return st;
    if (cfg->M == 0) return DENDSN_OK;
    if (!hidden || !weight || !labels || !loss || !lse)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "hidden, weight, labels, loss or lse is NULL");
    const bool bf = cfg->x_dtype == DENDSN_BF16, i64 = cfg->labels_dtype == DENDSN_I64;
    if (!seq_aligned(hidden, bf ? 2 : 4) || !seq_aligned(weight, bf ? 2 : 4) || !seq_aligned(labels, i64 ? 8 : 4) ||
        !seq_aligned(loss, 4) || !seq_aligned(lse, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "a tensor is misaligned");
    if (pl.fwd && !scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 256-byte aligned");
    Args a{};
    a.hidden = hidden;
    a.weight = weight;
    a.labels = labels;
    a.ignore = cfg->ignore_index;
    a.M = cfg->M;
    a.V = cfg->V;
    a.D = cfg->D;
    a.loss = loss;
    a.lse = lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = bf ? (i64 ? run_forward<__nv_bfloat16, int64_t>(a, s) : run_forward<__nv_bfloat16, int32_t>(a, s))
                       : (i64 ? run_forward<float, int64_t>(a, s) : run_forward<float, int32_t>(a, s));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "xent forward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

dendsn_status dendsn_xent_backward(const dendsn_xent_config *cfg, const void *hidden, const void *weight,
                                   const void *labels, const float *lse, const float *grad_loss,
                                   void *grad_hidden, void *grad_weight, void *scratch, void *stream) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
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
    if (pl.bwd && !scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 256-byte aligned");
    Args a{};
    a.hidden = hidden;
    a.weight = weight;
    a.labels = labels;
    a.ignore = cfg->ignore_index;
    a.M = cfg->M;
    a.V = cfg->V;
    a.D = cfg->D;
    a.lse_in = lse;
    a.gloss = grad_loss;
    a.gh = grad_hidden;
    a.gw = grad_weight;
    a.gh32 = static_cast<float *>(scratch);
    a.G = reinterpret_cast<float *>(static_cast<char *>(scratch) + pl.gh32);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int launches = 0;
    cudaError_t e = bf ? (i64 ? run_backward<__nv_bfloat16, int64_t>(a, s, &launches)
                              : run_backward<__nv_bfloat16, int32_t>(a, s, &launches))
                       : (i64 ? run_backward<float, int64_t>(a, s, &launches)
                              : run_backward<float, int32_t>(a, s, &launches));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "xent backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(launches);
    return DENDSN_OK;
}

}  // extern "C"
