// Embedding lookup with scaling (forward) and its gradient: out[i] = scale * table[ids[i]],
// grad_table[v] = scale * sum of grad_out[i] over ids[i] = v in ascending i.
#include <cuda_bf16.h>

#include "seq_common.h"

namespace dendsn {
namespace {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// One block per token.
template <typename T, typename I>
__global__ void embed_forward_kernel(const T *table, const I *ids, T *out, int64_t V, int64_t D,
                                     int64_t pad, float scale) {
    const int64_t i = blockIdx.x;
    const int64_t id = ids[i];
    for (int64_t d = threadIdx.x; d < D; d += blockDim.x) {
        float v = __int_as_float(0x7fffffff);
        if (pad >= 0 && id == pad) v = 0.f;
        else if (id >= 0 && id < V) v = scale * to_f<T>(table[id * D + d]);
        out[i * D + d] = from_f<T>(v);
    }
}

// One block per vocabulary row: scans all the ids, keeps the positions that match in order
// in shared memory, 256 ids at a time, and adds up their gradient rows.
template <typename T, typename I>
__global__ void __launch_bounds__(256) embed_backward_kernel(const I *ids, const T *grad, T *gtable,
                                                             int64_t n, int64_t D, int64_t pad,
                                                             float scale) {
    __shared__ int list[256];
    __shared__ int wcount[8];
    const int64_t v = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t d0 = 0; d0 < D; d0 += 256) {
        const int64_t d = d0 + threadIdx.x;
        float sum = 0.f;
        for (int64_t i0 = 0; i0 < n && v != pad; i0 += 256) {
            const int64_t i = i0 + threadIdx.x;
            const bool hit = i < n && (int64_t)ids[i] == v;
            const unsigned m = __ballot_sync(0xffffffffu, hit);
            if (lane == 0) wcount[warp] = __popc(m);
            __syncthreads();
            int base = 0, total = 0;
            for (int w = 0; w < 8; ++w) {
                if (w < warp) base += wcount[w];
                total += wcount[w];
            }
            if (hit) list[base + __popc(m & ((1u << lane) - 1))] = threadIdx.x;
            __syncthreads();
            if (d < D)
                for (int k = 0; k < total; ++k) sum += to_f<T>(grad[(i0 + list[k]) * D + d]);
            __syncthreads();
        }
        if (d < D) gtable[v * D + d] = from_f<T>(sum * scale);
    }
}

struct Plan {
    size_t scratch = 0;
};

dendsn_status make_plan(const dendsn_embed_config *cfg, Plan *pl) {
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->n < 0 || cfg->V < 1 || cfg->D < 1)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad size (n=%lld V=%d D=%d)", (long long)cfg->n, cfg->V, cfg->D);
    if (cfg->n > INT32_MAX) return seq_fail(DENDSN_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad x_dtype %d", cfg->x_dtype);
    if (cfg->ids_dtype != DENDSN_I32 && cfg->ids_dtype != DENDSN_I64)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad ids_dtype %d", cfg->ids_dtype);
    pl->scratch = 0;
    return DENDSN_OK;
}

template <typename T, typename I>
cudaError_t run_forward(const dendsn_embed_config &c, const void *table, const void *ids, void *out,
                        cudaStream_t s) {
    embed_forward_kernel<T, I><<<(unsigned)c.n, 256, 0, s>>>(
        static_cast<const T *>(table), static_cast<const I *>(ids), static_cast<T *>(out), c.V, c.D,
        c.padding_id, c.scale);
    return cudaGetLastError();
}

template <typename T, typename I>
cudaError_t run_backward(const dendsn_embed_config &c, const void *ids, const void *grad, void *gtable,
                         cudaStream_t s) {
    embed_backward_kernel<T, I><<<(unsigned)c.V, 256, 0, s>>>(
        static_cast<const I *>(ids), static_cast<const T *>(grad), static_cast<T *>(gtable), c.n, c.D,
        c.padding_id, c.scale);
    return cudaGetLastError();
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_embed_workspace_size(const dendsn_embed_config *cfg, size_t *scratch_bytes) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
    if (st != DENDSN_OK) return st;
    if (scratch_bytes) *scratch_bytes = pl.scratch;
    return DENDSN_OK;
}

dendsn_status dendsn_embed_forward(const dendsn_embed_config *cfg, const void *table, const void *ids,
                                   void *out, void *stream) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
    if (st != DENDSN_OK) return st;
    if (cfg->n == 0) return DENDSN_OK;
    if (!table || !ids || !out) return seq_fail(DENDSN_ERR_INVALID_ARG, "table, ids or out is NULL");
    const bool bf = cfg->x_dtype == DENDSN_BF16, i64 = cfg->ids_dtype == DENDSN_I64;
    const size_t sx = bf ? 2 : 4;
    if (!seq_aligned(table, sx) || !seq_aligned(out, sx) || !seq_aligned(ids, i64 ? 8 : 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "table, ids or out misaligned");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = bf ? (i64 ? run_forward<__nv_bfloat16, int64_t>(*cfg, table, ids, out, s)
                              : run_forward<__nv_bfloat16, int32_t>(*cfg, table, ids, out, s))
                       : (i64 ? run_forward<float, int64_t>(*cfg, table, ids, out, s)
                              : run_forward<float, int32_t>(*cfg, table, ids, out, s));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "embed forward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

dendsn_status dendsn_embed_backward(const dendsn_embed_config *cfg, const void *ids, const void *grad_out,
                                    void *grad_table, void *scratch, void *stream) {
    Plan pl;
    dendsn_status st = make_plan(cfg, &pl);
    if (st != DENDSN_OK) return st;
    if (!grad_table) return seq_fail(DENDSN_ERR_INVALID_ARG, "grad_table is NULL");
    if (cfg->n > 0 && (!ids || !grad_out)) return seq_fail(DENDSN_ERR_INVALID_ARG, "ids or grad_out is NULL");
    const bool bf = cfg->x_dtype == DENDSN_BF16, i64 = cfg->ids_dtype == DENDSN_I64;
    const size_t sx = bf ? 2 : 4;
    if (!seq_aligned(grad_out, sx) || !seq_aligned(grad_table, sx) || !seq_aligned(ids, i64 ? 8 : 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "ids, grad_out or grad_table misaligned");
    if (pl.scratch && !scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 16)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 16-byte aligned");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = bf ? (i64 ? run_backward<__nv_bfloat16, int64_t>(*cfg, ids, grad_out, grad_table, s)
                              : run_backward<__nv_bfloat16, int32_t>(*cfg, ids, grad_out, grad_table, s))
                       : (i64 ? run_backward<float, int64_t>(*cfg, ids, grad_out, grad_table, s)
                              : run_backward<float, int32_t>(*cfg, ids, grad_out, grad_table, s));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "embed backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

}  // extern "C"
