// Gated compartment scan: h[t] = a[t] h[t-1] + u[t] with an input-dependent decay a, and its
// backward. State in float32.
#include <cuda_bf16.h>

#include "seq_common.h"

namespace dendsn {
namespace {

constexpr int kInterval = 64;     // steps between checkpoints

struct ScanArgs {
    int64_t M;                    // channels B * N
    int32_t T, N;
    int64_t st, sb;               // element strides of a step and of a sample
    int64_t ft, fb;               // strides of the start flags
    const void *x, *gate, *gh;
    const uint8_t *starts;
    const float *h0, *glast;
    void *h, *gx, *gg;
    float *last, *saved, *gh0;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// a and 1 - a; the complement of a logistic decay is formed as 1 / (1 + exp(g)), which
// keeps its relative precision where a is close to 1.
template <bool LOGIT> __device__ __forceinline__ void decay_of(float g, float &a, float &na) {
    if (LOGIT) {
        a = 1.f / (1.f + expf(-g));
        na = 1.f / (1.f + expf(g));
    } else {
        a = g;
        na = 1.f - g;
    }
}

// One thread per channel, step by step.
template <typename XT, bool LOGIT, bool MIX>
__global__ void scan_forward_kernel(const ScanArgs A) {
    const int64_t m = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (m >= A.M) return;
    const int64_t b = m / A.N, off = b * A.sb + m % A.N;
    const XT *x = static_cast<const XT *>(A.x) + off, *g = static_cast<const XT *>(A.gate) + off;
    XT *h = static_cast<XT *>(A.h) + off;
    float v = A.h0 ? A.h0[m] : 0.f;
    for (int t = 0; t < A.T; ++t) {
        float a, na;
        decay_of<LOGIT>(to_f<XT>(g[t * A.st]), a, na);
        const float xv = to_f<XT>(x[t * A.st]);
        const float u = MIX ? na * xv : xv;
        const bool start = A.starts && A.starts[t * A.ft + b * A.fb];
        v = start ? u : fmaf(a, v, u);
        h[t * A.st] = from_f<XT>(v);
        if (A.saved && (t + 1) % kInterval == 0 && t + 1 < A.T)
            A.saved[(int64_t)(t / kInterval) * A.M + m] = v;
    }
    if (A.last) A.last[m] = v;
}

template <typename XT, bool LOGIT, bool MIX>
__global__ void scan_backward_kernel(const ScanArgs A) {
    const int64_t m = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (m >= A.M) return;
    const int64_t b = m / A.N, off = b * A.sb + m % A.N;
    const XT *x = static_cast<const XT *>(A.x) + off, *g = static_cast<const XT *>(A.gate) + off;
    const XT *gh = static_cast<const XT *>(A.gh) + off;
    XT *gx = static_cast<XT *>(A.gx) + off, *gg = static_cast<XT *>(A.gg) + off;
    float before[kInterval];      // h[t-1] of the chunk's steps
    float mu = A.glast ? A.glast[m] : 0.f;
    for (int c = (A.T + kInterval - 1) / kInterval - 1; c >= 0; --c) {
        const int t0 = c * kInterval, t1 = min(A.T, t0 + kInterval);
        float v = c ? A.saved[(int64_t)(c - 1) * A.M + m] : A.h0 ? A.h0[m] : 0.f;
        for (int t = t0; t < t1; ++t) {
            before[t - t0] = v;
            float a, na;
            decay_of<LOGIT>(to_f<XT>(g[t * A.st]), a, na);
            const float xv = to_f<XT>(x[t * A.st]);
            const float u = MIX ? na * xv : xv;
            const bool start = A.starts && A.starts[t * A.ft + b * A.fb];
            v = start ? u : fmaf(a, v, u);
        }
        for (int t = t1 - 1; t >= t0; --t) {
            float a, na;
            decay_of<LOGIT>(to_f<XT>(g[t * A.st]), a, na);
            const float xv = to_f<XT>(x[t * A.st]);
            const bool start = A.starts && A.starts[t * A.ft + b * A.fb];
            const float lam = to_f<XT>(gh[t * A.st]) + mu;
            const float hp = start ? 0.f : before[t - t0];
            const float ga = lam * (MIX ? hp - xv : hp);
            gx[t * A.st] = from_f<XT>(MIX ? lam * na : lam);
            gg[t * A.st] = from_f<XT>(LOGIT ? ga * a * na : ga);
            mu = start ? 0.f : a * lam;
        }
    }
    if (A.gh0) A.gh0[m] = mu;
}

dendsn_status check(const dendsn_scan_config *cfg, size_t *saved) {
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->T < 0 || cfg->B < 0 || cfg->N < 0)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "negative size (T=%d B=%d N=%d)", cfg->T, cfg->B, cfg->N);
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad x_dtype %d", cfg->x_dtype);
    if ((cfg->gate & ~1) || (cfg->mix & ~1) || (cfg->layout & ~1))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "enum field out of range");
    const int64_t M = (int64_t)cfg->B * cfg->N;
    if (M > (int64_t)INT32_MAX) return seq_fail(DENDSN_ERR_UNSUPPORTED, "too many channels");
    const int64_t n = cfg->T > kInterval ? (cfg->T + kInterval - 1) / kInterval - 1 : 0;
    *saved = ((size_t)n * M * 4 + 15) / 16 * 16;
    return DENDSN_OK;
}

ScanArgs make_args(const dendsn_scan_config &c) {
    ScanArgs a{};
    a.M = (int64_t)c.B * c.N;
    a.T = c.T;
    a.N = c.N;
    const bool batch = c.layout == DENDSN_BATCH_FIRST;
    a.st = batch ? c.N : a.M;
    a.sb = batch ? (int64_t)c.T * c.N : c.N;
    a.ft = batch ? 1 : c.B;
    a.fb = batch ? c.T : 1;
    return a;
}

template <typename XT, bool LOGIT, bool MIX>
cudaError_t launch(bool forward, const ScanArgs &a, cudaStream_t s) {
    const unsigned blocks = (unsigned)((a.M + 127) / 128);
    if (forward) scan_forward_kernel<XT, LOGIT, MIX><<<blocks, 128, 0, s>>>(a);
    else scan_backward_kernel<XT, LOGIT, MIX><<<blocks, 128, 0, s>>>(a);
    return cudaGetLastError();
}

template <typename XT>
cudaError_t dispatch(const dendsn_scan_config &c, bool forward, const ScanArgs &a, cudaStream_t s) {
    if (c.gate == DENDSN_GATE_LOGIT)
        return c.mix ? launch<XT, true, true>(forward, a, s) : launch<XT, true, false>(forward, a, s);
    return c.mix ? launch<XT, false, true>(forward, a, s) : launch<XT, false, false>(forward, a, s);
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_scan_workspace_size(const dendsn_scan_config *cfg, size_t *saved_bytes) {
    size_t saved = 0;
    dendsn_status st = check(cfg, &saved);
    if (st != DENDSN_OK) return st;
    if (saved_bytes) *saved_bytes = saved;
    return DENDSN_OK;
}

dendsn_status dendsn_scan_forward(const dendsn_scan_config *cfg, const void *x, const void *gate,
                                  const uint8_t *starts, const float *h0, void *h, float *h_last,
                                  void *saved, void *stream) {
    size_t bytes = 0;
    dendsn_status st = check(cfg, &bytes);
    if (st != DENDSN_OK) return st;
    ScanArgs a = make_args(*cfg);
    if (a.M == 0) return DENDSN_OK;
    if (a.T > 0 && (!x || !gate || !h)) return seq_fail(DENDSN_ERR_INVALID_ARG, "x, gate or h is NULL");
    const size_t sx = cfg->x_dtype == DENDSN_BF16 ? 2 : 4;
    if (!seq_aligned(x, sx) || !seq_aligned(gate, sx) || !seq_aligned(h, sx) || !seq_aligned(h0, 4) ||
        !seq_aligned(h_last, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "x, gate, h, h0 or h_last misaligned");
    if (!seq_aligned(saved, 16)) return seq_fail(DENDSN_ERR_MISALIGNED, "saved must be 16-byte aligned");
    a.x = x;
    a.gate = gate;
    a.starts = starts;
    a.h0 = h0;
    a.h = h;
    a.last = h_last;
    a.saved = bytes ? static_cast<float *>(saved) : nullptr;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = sx == 2 ? dispatch<__nv_bfloat16>(*cfg, true, a, s) : dispatch<float>(*cfg, true, a, s);
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "scan forward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

dendsn_status dendsn_scan_backward(const dendsn_scan_config *cfg, const void *x, const void *gate,
                                   const uint8_t *starts, const float *h0, const void *grad_h,
                                   const float *grad_last, const void *saved, void *grad_x,
                                   void *grad_gate, float *grad_h0, void *stream) {
    size_t bytes = 0;
    dendsn_status st = check(cfg, &bytes);
    if (st != DENDSN_OK) return st;
    ScanArgs a = make_args(*cfg);
    if (a.M == 0) return DENDSN_OK;
    if (a.T > 0 && (!x || !gate || !grad_h || !grad_x || !grad_gate))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "x, gate, grad_h, grad_x or grad_gate is NULL");
    if (bytes && !saved)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "T=%d needs the forward's saved states", cfg->T);
    const size_t sx = cfg->x_dtype == DENDSN_BF16 ? 2 : 4;
    if (!seq_aligned(x, sx) || !seq_aligned(gate, sx) || !seq_aligned(grad_h, sx) || !seq_aligned(h0, 4) ||
        !seq_aligned(grad_last, 4) || !seq_aligned(grad_x, sx) || !seq_aligned(grad_gate, sx) ||
        !seq_aligned(grad_h0, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "a tensor is misaligned");
    if (!seq_aligned(saved, 16)) return seq_fail(DENDSN_ERR_MISALIGNED, "saved must be 16-byte aligned");
    a.x = x;
    a.gate = gate;
    a.starts = starts;
    a.h0 = h0;
    a.gh = grad_h;
    a.glast = grad_last;
    a.saved = static_cast<float *>(const_cast<void *>(saved));
    a.gx = grad_x;
    a.gg = grad_gate;
    a.gh0 = grad_h0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = sx == 2 ? dispatch<__nv_bfloat16>(*cfg, false, a, s) : dispatch<float>(*cfg, false, a, s);
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "scan backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(1);
    return DENDSN_OK;
}

}  // extern "C"
