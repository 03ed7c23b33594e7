// Gated compartment scan: h[t] = a[t] h[t-1] + u[t] with an input-dependent decay a, and its
// backward. State in float32.
//
// Split. A thread owns VEC neighbouring channels and a segment of S steps; the eight warps of
// a block stand side by side in time (WT of them) and in channels, and the blocks of a cluster
// follow one another in time. A segment of the recurrence is the map h -> A h + B with
// A = prod a, B = its end from a zero state, so a pass is: load the segment into registers,
// form (A, B), fold the maps of the earlier segments over the state (shared memory within the
// block, distributed shared memory between the blocks of the cluster), then run the segment
// from its true state and write. Every element is read and written once; the loads of the next
// pass are issued before the fold, so that its barriers overlap with memory.
// A start makes its segment's map constant; that is kept as a flag and selected, not
// multiplied by zero, so that what came before it cannot leak as NaN.
//
// The backward runs the passes from the last step to the first with the map
// mu -> A mu + L of mu[t] = a[t] (grad_h[t] + mu[t+1]), and recomputes h from x, gate and the
// state kept every 64 steps: three arrays read and two written, against four read if h were
// kept, and no rounding of h to the output's type enters the gradient.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

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
    int32_t WT, WC, CT;           // warps along time and channels, blocks of a cluster
};

// VEC elements of a row, loaded and stored at once, held as they are until they are used.
template <typename XT, int VEC> struct Row;
template <int VEC> struct Row<float, VEC> {
    using Raw = typename std::conditional<VEC == 4, float4,
                typename std::conditional<VEC == 2, float2, float>::type>::type;
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[VEC]) {
        if constexpr (VEC == 4) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
        else if constexpr (VEC == 2) { v[0] = r.x; v[1] = r.y; }
        else v[0] = r;
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[VEC]) {
        if constexpr (VEC == 4) return make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (VEC == 2) return make_float2(v[0], v[1]);
        else return v[0];
    }
};
template <int VEC> struct Row<__nv_bfloat16, VEC> {
    using Raw = typename std::conditional<VEC == 4, uint2,
                typename std::conditional<VEC == 2, uint32_t, uint16_t>::type>::type;
    static __device__ __forceinline__ float lo(uint32_t q) { return __uint_as_float(q << 16); }
    static __device__ __forceinline__ float hi(uint32_t q) { return __uint_as_float(q & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[VEC]) {
        if constexpr (VEC == 4) { v[0] = lo(r.x); v[1] = hi(r.x); v[2] = lo(r.y); v[3] = hi(r.y); }
        else if constexpr (VEC == 2) { v[0] = lo(r); v[1] = hi(r); }
        else v[0] = lo(r);
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[VEC]) {
        if constexpr (VEC == 4) return make_uint2(two(v[0], v[1]), two(v[2], v[3]));
        else if constexpr (VEC == 2) return two(v[0], v[1]);
        else {
            const __nv_bfloat16 h = __float2bfloat16_rn(v[0]);
            return *reinterpret_cast<const uint16_t *>(&h);
        }
    }
};

template <typename XT, int VEC>
__device__ __forceinline__ typename Row<XT, VEC>::Raw load_row(const void *p, int64_t at) {
    return __ldcs(reinterpret_cast<const typename Row<XT, VEC>::Raw *>(static_cast<const XT *>(p) + at));
}
template <typename XT, int VEC>
__device__ __forceinline__ void store_row(void *p, int64_t at, const float (&v)[VEC]) {
    __stcs(reinterpret_cast<typename Row<XT, VEC>::Raw *>(static_cast<XT *>(p) + at), Row<XT, VEC>::pack(v));
}

// a and 1 - a. Of a logistic decay both come from e = exp(-|g|), each with its own relative
// precision: 1 / (1 + e) and e / (1 + e). bfloat16 gates take the hardware's exponential and
// reciprocal (about 2^-21 relative), float32 gates the correctly rounded forms.
template <typename XT, bool LOGIT> __device__ __forceinline__ void decay_of(float g, float &a, float &na) {
    if constexpr (LOGIT) {
        constexpr bool fast = sizeof(XT) == 2;
        const float e = fast ? __expf(-fabsf(g)) : expf(-fabsf(g));
        const float r = fast ? __fdividef(1.f, 1.f + e) : 1.f / (1.f + e);
        const float q = e * r;
        a = g >= 0.f ? r : q;
        na = g >= 0.f ? q : r;
        if (g != g) a = na = g;
    } else {
        a = g;
        na = 1.f - g;
    }
}

// A h + B of a segment's map over a state, B alone where the segment has a start; a state of
// zero stays zero under a product of decays that overflowed.
__device__ __forceinline__ float map_over(float A, float B, int cut, float h) {
    return cut || h == 0.f ? B : fmaf(A, h, B);
}

// The maps of the block's warps, of the block as a whole (two buffers, read by the cluster's
// other blocks) and of the cluster's blocks.
template <int VEC> struct ScanShared {
    float A[8][32][VEC], B[8][32][VEC];
    float tA[2][32][VEC], tB[2][32][VEC];
    float rA[2][8][32][VEC], rB[2][8][32][VEC];
    int cut[8][32], tcut[2][32], rcut[2][8][32];
};

// Folds the segment maps over `carry`, the state at the pass's first step (the last one, when
// REVERSE). Returns in `in` the state before this warp's segment; advances carry by the pass.
template <int VEC, bool CL, bool REVERSE>
__device__ __forceinline__ void fold(ScanShared<VEC> &sh, const ScanArgs &P, int wt, int wc, int lane,
                                     int rank, int pass, const float (&A)[VEC], const float (&B)[VEC],
                                     int cut, float (&carry)[VEC], float (&in)[VEC]) {
    const int w0 = wc * P.WT;
    if (!CL || pass) __syncthreads();         // the maps of the pass before are read
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        sh.A[w0 + wt][lane][e] = A[e];
        sh.B[w0 + wt][lane][e] = B[e];
    }
    sh.cut[w0 + wt][lane] = cut;
    __syncthreads();
    if constexpr (CL) {
        namespace cg = cooperative_groups;
        cg::cluster_group cluster = cg::this_cluster();
        const int buf = pass & 1;
        if (wt == 0) {                        // the block's own map
            float tA[VEC], tB[VEC];
            int tc = 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) { tA[e] = 1.f; tB[e] = 0.f; }
            for (int i = 0; i < P.WT; ++i) {
                const int w = w0 + (REVERSE ? P.WT - 1 - i : i);
                const int c = sh.cut[w][lane];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float a = sh.A[w][lane][e];
                    tB[e] = map_over(a, sh.B[w][lane][e], c, tB[e]);
                    tA[e] *= a;
                }
                tc |= c;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                sh.tA[buf][lane][e] = tA[e];
                sh.tB[buf][lane][e] = tB[e];
            }
            sh.tcut[buf][lane] = tc;
        }
        cluster.sync();
        const int warp = threadIdx.x >> 5;
        if (warp < P.CT) {                    // each warp fetches one block's map
            const ScanShared<VEC> *from = cluster.map_shared_rank(&sh, warp);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                sh.rA[buf][warp][lane][e] = from->tA[buf][lane][e];
                sh.rB[buf][warp][lane][e] = from->tB[buf][lane][e];
            }
            sh.rcut[buf][warp][lane] = from->tcut[buf][lane];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < VEC; ++e) in[e] = carry[e];
        for (int i = 0; i < P.CT; ++i) {
            const int r = REVERSE ? P.CT - 1 - i : i;
            if (r == rank)
#pragma unroll
                for (int e = 0; e < VEC; ++e) in[e] = carry[e];
            const int c = sh.rcut[buf][r][lane];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                carry[e] = map_over(sh.rA[buf][r][lane][e], sh.rB[buf][r][lane][e], c, carry[e]);
        }
        for (int i = 0; i < (REVERSE ? P.WT - 1 - wt : wt); ++i) {
            const int w = w0 + (REVERSE ? P.WT - 1 - i : i);
            const int c = sh.cut[w][lane];
#pragma unroll
            for (int e = 0; e < VEC; ++e) in[e] = map_over(sh.A[w][lane][e], sh.B[w][lane][e], c, in[e]);
        }
    } else {
        for (int i = 0; i < P.WT; ++i) {
            const int k = REVERSE ? P.WT - 1 - i : i, w = w0 + k;
            if (k == wt)
#pragma unroll
                for (int e = 0; e < VEC; ++e) in[e] = carry[e];
            const int c = sh.cut[w][lane];
#pragma unroll
            for (int e = 0; e < VEC; ++e) carry[e] = map_over(sh.A[w][lane][e], sh.B[w][lane][e], c, carry[e]);
        }
    }
}

template <bool CL> __device__ __forceinline__ void leave_cluster() {
    if constexpr (CL) cooperative_groups::this_cluster().sync();   // no block's maps are still read
}

template <typename XT, int VEC, int S, bool LOGIT, bool MIX, bool CL>
__global__ void __launch_bounds__(256) scan_forward_kernel(const ScanArgs P) {
    using R = Row<XT, VEC>;
    __shared__ ScanShared<VEC> sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wt = warp % P.WT, wc = warp / P.WT;
    const int rank = CL ? blockIdx.x % P.CT : 0;
    const int64_t m = ((int64_t)(CL ? blockIdx.x / P.CT : blockIdx.x) * P.WC * 32 + wc * 32 + lane) * VEC;
    const bool on = m < P.M;
    const int64_t b = on ? m / P.N : 0, off = on ? b * P.sb + m % P.N : 0;
    float carry[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) carry[e] = on && P.h0 ? P.h0[m + e] : 0.f;
    if (P.T == 0) {
        if (on && wt == 0 && rank == 0 && P.last)
            for (int e = 0; e < VEC; ++e) P.last[m + e] = carry[e];
        leave_cluster<CL>();
        return;
    }
    const int span = P.WT * S, step = span * (CL ? P.CT : 1);
    typename R::Raw gr[S], xr[S];
    uint32_t st = 0;
    auto fetch = [&](int t0) {
        st = 0;
        if (!on) return;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (t0 + s < P.T) {
                gr[s] = load_row<XT, VEC>(P.gate, off + (t0 + s) * P.st);
                xr[s] = load_row<XT, VEC>(P.x, off + (t0 + s) * P.st);
            }
        if (P.starts) {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 + s < P.T && P.starts[(t0 + s) * P.ft + b * P.fb]) st |= 1u << s;
        }
    };
    int t0 = rank * span + wt * S;
    fetch(t0);
    for (int pass = 0; pass * (int64_t)step < P.T; ++pass) {
        float a[S][VEC], u[S][VEC], A[VEC], B[VEC], h[VEC];
        const uint32_t cut = st;
#pragma unroll
        for (int e = 0; e < VEC; ++e) { A[e] = 1.f; B[e] = 0.f; }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (on && t0 + s < P.T) {
                float g[VEC], x[VEC];
                R::unpack(gr[s], g);
                R::unpack(xr[s], x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float na;
                    decay_of<XT, LOGIT>(g[e], a[s][e], na);
                    u[s][e] = MIX ? na * x[e] : x[e];
                    A[e] *= a[s][e];
                    B[e] = cut >> s & 1 ? u[s][e] : fmaf(a[s][e], B[e], u[s][e]);
                }
            }
        }
        const int t1 = t0;
        t0 += step;
        fetch(t0);
        fold<VEC, CL, false>(sh, P, wt, wc, lane, rank, pass, A, B, cut != 0, carry, h);
        if (on && t1 < P.T) {
            if (P.saved && t1 && t1 % kInterval == 0)
#pragma unroll
                for (int e = 0; e < VEC; ++e) P.saved[(int64_t)(t1 / kInterval - 1) * P.M + m + e] = h[e];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if (t1 + s < P.T) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        h[e] = cut >> s & 1 ? u[s][e] : fmaf(a[s][e], h[e], u[s][e]);
                    store_row<XT, VEC>(P.h, off + (t1 + s) * P.st, h);
                }
            }
            if (P.last && P.T - t1 <= S)
#pragma unroll
                for (int e = 0; e < VEC; ++e) P.last[m + e] = h[e];
        }
    }
    leave_cluster<CL>();
}

template <typename XT, int VEC, int S, bool LOGIT, bool MIX, bool CL>
__global__ void __launch_bounds__(256) scan_backward_kernel(const ScanArgs P) {
    using R = Row<XT, VEC>;
    __shared__ ScanShared<VEC> sh;
    __shared__ float fA[8][32][VEC], fB[8][32][VEC];     // the forward maps of the block's warps
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wt = warp % P.WT, wc = warp / P.WT;
    const int rank = CL ? blockIdx.x % P.CT : 0;
    const int64_t m = ((int64_t)(CL ? blockIdx.x / P.CT : blockIdx.x) * P.WC * 32 + wc * 32 + lane) * VEC;
    const bool on = m < P.M;
    const int64_t b = on ? m / P.N : 0, off = on ? b * P.sb + m % P.N : 0;
    float carry[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) carry[e] = on && P.glast ? P.glast[m + e] : 0.f;
    if (P.T == 0) {
        if (on && wt == 0 && rank == 0 && P.gh0)
            for (int e = 0; e < VEC; ++e) P.gh0[m + e] = carry[e];
        leave_cluster<CL>();
        return;
    }
    const int span = P.WT * S, step = span * (CL ? P.CT : 1);
    const int passes = (P.T - 1) / step + 1;
    typename R::Raw gr[S], xr[S], lr[S];
    uint32_t st = 0;
    float start[VEC];                                    // h before the block's first step
    auto fetch = [&](int t0) {
        st = 0;
        if (!on || t0 < 0) return;
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (t0 + s < P.T) {
                gr[s] = load_row<XT, VEC>(P.gate, off + (t0 + s) * P.st);
                xr[s] = load_row<XT, VEC>(P.x, off + (t0 + s) * P.st);
                lr[s] = load_row<XT, VEC>(P.gh, off + (t0 + s) * P.st);
            }
        if (P.starts) {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 + s < P.T && P.starts[(t0 + s) * P.ft + b * P.fb]) st |= 1u << s;
        }
        const int tb = t0 - wt * S;                      // a multiple of the interval, or 0
        if (tb < P.T) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                start[e] = tb ? P.saved[(int64_t)(tb / kInterval - 1) * P.M + m + e] : P.h0 ? P.h0[m + e] : 0.f;
        }
    };
    int t0 = (passes - 1) * step + rank * span + wt * S;
#pragma unroll
    for (int e = 0; e < VEC; ++e) start[e] = 0.f;
    fetch(t0);
    for (int pass = 0; pass < passes; ++pass) {
        float a[S][VEC], x[S][VEC], g[S][VEC], gh[S][VEC], A[VEC], B[VEC], L[VEC], h[VEC], mu[VEC];
        const uint32_t cut = st;
        const int t1 = t0;
        auto live = [&](int s) { return on && t1 + s < P.T; };
#pragma unroll
        for (int e = 0; e < VEC; ++e) { A[e] = 1.f; B[e] = 0.f; L[e] = 0.f; }
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (live(s)) {
                R::unpack(gr[s], g[s]);
                R::unpack(xr[s], x[s]);
                R::unpack(lr[s], gh[s]);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float na;
                    decay_of<XT, LOGIT>(g[s][e], a[s][e], na);
                    if (LOGIT) g[s][e] = na;             // the gate itself is not needed again
                    const float u = MIX ? na * x[s][e] : x[s][e];
                    A[e] *= a[s][e];
                    B[e] = cut >> s & 1 ? u : fmaf(a[s][e], B[e], u);
                }
            }
#pragma unroll
        for (int s = S - 1; s >= 0; --s)
            if (live(s)) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) L[e] = cut >> s & 1 ? 0.f : a[s][e] * (gh[s][e] + L[e]);
            }
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[e] = start[e];
        t0 -= step;
        fetch(t0);
        if (pass) __syncthreads();
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            fA[warp][lane][e] = A[e];
            fB[warp][lane][e] = B[e];
        }
        fold<VEC, CL, true>(sh, P, wt, wc, lane, rank, pass, A, L, cut != 0, carry, mu);
        for (int i = 0; i < wt; ++i) {
            const int w = wc * P.WT + i;
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[e] = map_over(fA[w][lane][e], fB[w][lane][e], sh.cut[w][lane], h[e]);
        }
        float before[S][VEC];
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (live(s)) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const bool c = cut >> s & 1;
                    const float u = MIX ? (LOGIT ? g[s][e] : 1.f - a[s][e]) * x[s][e] : x[s][e];
                    before[s][e] = c ? 0.f : h[e];
                    h[e] = c ? u : fmaf(a[s][e], h[e], u);
                }
            }
#pragma unroll
        for (int s = S - 1; s >= 0; --s)
            if (live(s)) {
                float gx[VEC], gg[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float na = LOGIT ? g[s][e] : 1.f - a[s][e];
                    const float lam = gh[s][e] + mu[e];
                    const float ga = lam * (MIX ? before[s][e] - x[s][e] : before[s][e]);
                    gx[e] = MIX ? lam * na : lam;
                    gg[e] = LOGIT ? ga * a[s][e] * na : ga;
                    mu[e] = cut >> s & 1 ? 0.f : a[s][e] * lam;
                }
                store_row<XT, VEC>(P.gx, off + (t1 + s) * P.st, gx);
                store_row<XT, VEC>(P.gg, off + (t1 + s) * P.st, gg);
            }
        if (on && t1 == 0 && P.gh0)
#pragma unroll
            for (int e = 0; e < VEC; ++e) P.gh0[m + e] = mu[e];
    }
    leave_cluster<CL>();
}

dendsn_status check(const dendsn_scan_config *cfg, size_t *saved) {
    if (!cfg) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (cfg->T < 0 || cfg->B < 0 || cfg->N < 0)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "negative size (T=%d B=%d N=%d)", cfg->T, cfg->B, cfg->N);
    if (cfg->x_dtype != DENDSN_F32 && cfg->x_dtype != DENDSN_BF16)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "bad x_dtype %d", cfg->x_dtype);
    if ((cfg->gate & ~1) || (cfg->mix & ~1) || (cfg->layout & ~1))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "enum field out of range");
    if (cfg->T > 1 << 30) return seq_fail(DENDSN_ERR_UNSUPPORTED, "more than 2^30 steps");
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

// Blocks that keep the card busy: two for each of its 152 SMs.
constexpr int kBusy = 304;

// How a call is split. Time: as many of a block's eight warps as the steps fill, then blocks of
// a cluster while the channels alone give fewer than kBusy blocks.
struct Split {
    int WT, WC, CT;
    unsigned blocks;
};
Split split_of(const ScanArgs &a, int vec, int S) {
    Split p;
    p.WT = a.T > 4 * S ? 8 : a.T > 2 * S ? 4 : a.T > S ? 2 : 1;
    p.WC = 8 / p.WT;
    const int64_t width = (int64_t)p.WC * 32 * vec, groups = (a.M + width - 1) / width;
    p.CT = 1;
    while (p.CT < 8 && groups * p.CT < kBusy && a.T > p.WT * S * p.CT) p.CT *= 2;
    p.blocks = (unsigned)(groups * p.CT);
    return p;
}

template <typename XT, int VEC, int S, bool LOGIT, bool MIX, bool FWD>
cudaError_t launch(ScanArgs a, cudaStream_t s) {
    const Split p = split_of(a, VEC, S);
    a.WT = p.WT;
    a.WC = p.WC;
    a.CT = p.CT;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.blocks);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)p.CT;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.CT > 1 ? 1 : 0;
    if constexpr (FWD)
        return p.CT > 1 ? cudaLaunchKernelEx(&cfg, scan_forward_kernel<XT, VEC, S, LOGIT, MIX, true>, a)
                        : cudaLaunchKernelEx(&cfg, scan_forward_kernel<XT, VEC, S, LOGIT, MIX, false>, a);
    else
        return p.CT > 1 ? cudaLaunchKernelEx(&cfg, scan_backward_kernel<XT, VEC, S, LOGIT, MIX, true>, a)
                        : cudaLaunchKernelEx(&cfg, scan_backward_kernel<XT, VEC, S, LOGIT, MIX, false>, a);
}

template <typename XT, int VEC, bool LOGIT, bool MIX>
cudaError_t launch_vec(bool forward, const ScanArgs &a, cudaStream_t s) {
    return forward ? launch<XT, VEC, 8, LOGIT, MIX, true>(a, s) : launch<XT, VEC, 8, LOGIT, MIX, false>(a, s);
}

// Widest vector whose pieces lie within one sample's row and are aligned in every tensor.
template <typename XT, bool LOGIT, bool MIX>
cudaError_t launch_form(bool forward, const ScanArgs &a, cudaStream_t s) {
    auto fits = [&](int vec) {
        const size_t bytes = vec * sizeof(XT);
        return a.N % vec == 0 && seq_aligned(a.x, bytes) && seq_aligned(a.gate, bytes) && seq_aligned(a.h, bytes) &&
               seq_aligned(a.gh, bytes) && seq_aligned(a.gx, bytes) && seq_aligned(a.gg, bytes);
    };
    const int vec = fits(2) ? 2 : 1;
    return vec == 2 ? launch_vec<XT, 2, LOGIT, MIX>(forward, a, s) : launch_vec<XT, 1, LOGIT, MIX>(forward, a, s);
}

template <typename XT>
cudaError_t dispatch(const dendsn_scan_config &c, bool forward, const ScanArgs &a, cudaStream_t s) {
    if (c.gate == DENDSN_GATE_LOGIT)
        return c.mix ? launch_form<XT, true, true>(forward, a, s) : launch_form<XT, true, false>(forward, a, s);
    return c.mix ? launch_form<XT, false, true>(forward, a, s) : launch_form<XT, false, false>(forward, a, s);
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
