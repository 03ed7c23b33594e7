// Gated compartment scan: h[t] = a[t] h[t-1] + u[t] with an input-dependent decay a, and its
// backward. State in float32.
//
// Split. A thread owns a pair of neighbouring channels and a segment of S steps; the 256
// threads of a block are Q segments one after the other of 256 / Q pairs, and the blocks of a
// cluster follow one another in time. A segment of the recurrence is the map h -> A h + B with
// A = prod a, B = its end from a zero state, so a pass is: load the segment into registers,
// form (A, B), fold the maps of the earlier segments over the state (shared memory within the
// block, distributed shared memory between the blocks of the cluster), then run the segment
// from its true state and write. Every element is read and written once; the rows of the
// passes to come are copied to shared memory meanwhile (cp.async, 16 bytes a thread where rows
// are aligned), each warp its own segments, so that registers hold one segment only. Results go
// back through the same slots, to be written 16 bytes at a time.
// A start makes its segment's map constant; that is kept as a flag and selected, not
// multiplied by zero, so that what came before it cannot leak as NaN.
// Products of decays above 1 are kept as mantissa and exponent, so that they may leave float32 where
// the states do not (decays of at most 1 only pay for the look at them: 16384 steps of 1024 float32
// channels, forward and backward, 133 -> 138 us).
//
// The backward runs the passes from the last step to the first with the map
// mu -> A mu + L of mu[t] = a[t] (grad_h[t] + mu[t+1]), and recomputes h from x, gate and the
// state kept every 64 steps: three arrays read and two written, against four read if h were
// kept, and no rounding of h to the output's type enters the gradient.
//
// Bound: 6 (forward) and 10 bytes (backward) of a bfloat16 element against the instructions on
// it; the arithmetic runs on pairs (f32x2), which halves it. Measured, 2048 steps of 65536
// bfloat16 channels, logistic decays, sequence starts: forward 148 us (5.5 TB/s), backward 277 us
// (4.8 TB/s); their 1024 blocks are 3.4 rounds of the 304 that fit.
// 16384 steps of 1024 float32 channels: 49 us (4.1 TB/s) and 98 us (3.4 TB/s), 256 blocks in
// clusters of 8 along time. One step of 262144 bfloat16 channels: 8 us, a launch and one pass's latency.
#include <cuda_bf16.h>

#include <algorithm>

#include "pairs.cuh"
#include "scan_fold.cuh"
#include "seq_common.h"

namespace dendsn {
namespace {

constexpr int kInterval = 64;     // steps between checkpoints
// Passes in shared memory at once. Two blocks of an SM have to fit (a cluster of 8 that finds one
// block an SM waits for a second round: 16384 steps of 1024 float32 channels 51 -> 150 us with a
// third stage).
template <typename XT> constexpr int kForwardStages = sizeof(XT) == 2 ? 4 : 2;
template <typename XT> constexpr int kBackwardStages = sizeof(XT) == 2 ? 3 : 2;

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
    int32_t Q, CT;                // segments of a block, blocks of a cluster
    int32_t PN;                   // pairs of a sample
    int64_t pairs;                // in all
};

// One element and a pair of elements as they lie in memory.
template <typename XT> struct Elem;
template <> struct Elem<float> {
    using One = float;
    using Pair = float2;
    static __device__ __forceinline__ Pair pair(One a, One b) { return make_float2(a, b); }
    static __device__ __forceinline__ One first(Pair p) { return p.x; }
    static __device__ __forceinline__ One second(Pair p) { return p.y; }
    static __device__ __forceinline__ F2 unpack(Pair p) { return F2(p.x, p.y); }
    static __device__ __forceinline__ Pair pack(F2 v) { return make_float2(v.x(), v.y()); }
};
template <> struct Elem<__nv_bfloat16> {
    using One = uint16_t;
    using Pair = uint32_t;
    static __device__ __forceinline__ Pair pair(One a, One b) { return (uint32_t)a | (uint32_t)b << 16; }
    static __device__ __forceinline__ One first(Pair p) { return (One)p; }
    static __device__ __forceinline__ One second(Pair p) { return (One)(p >> 16); }
    static __device__ __forceinline__ F2 unpack(Pair p) {
        return F2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u));
    }
    static __device__ __forceinline__ Pair pack(F2 v) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v.x(), v.y());
        return *reinterpret_cast<const uint32_t *>(&h);
    }
};

// a and 1 - a. Of a logistic decay both come from e = exp(-g), each with its own relative
// precision: 1 / (1 + e) and e / (1 + e), from the hardware's exponential and reciprocal, within
// 2^-21 at every gate (measured 2^-22.2 at most, all bfloat16 gates up to 79 of 0).
// bfloat16 gates are kept above -80, where a is below 2e-35 and e still finite, and below 101, where
// e is 0. Their 8 bits times the first 16 of log2(e), 1.44268798828125, are exact; the rest of it
// is multiplied in behind the exponential (left out and rounded instead: 2^-18.2 at 79).
// float32 gates have the product's rounding and the rest of log2(e) multiplied in, and a Newton
// step; beyond 88.5 of 0 the smaller of the two is flushed to 0.
template <bool LOGIT> __device__ __forceinline__ void decay_of(uint32_t raw, F2 &a, F2 &na) {
    if constexpr (LOGIT) {
        uint32_t g;
        asm("max.NaN.bf16x2 %0, %1, %2;\n\tmin.NaN.bf16x2 %0, %0, %3;" : "=&r"(g) : "r"(raw), "r"(0xC2A0C2A0u), "r"(0x42CA42CAu));
        const F2 v = Elem<__nv_bfloat16>::unpack(g), t = mul(v, both(-1.44268798828125f));
        F2 e(exp2_fast(t.x()), exp2_fast(t.y()));
        e = fma(e, mul(v, both(-4.88849420e-6f)), e);
        const F2 d = add(e, both(1.f));
        a = F2(rcp_fast(d.x()), rcp_fast(d.y()));
        na = mul(e, a);
    } else {
        a = Elem<__nv_bfloat16>::unpack(raw);
        na = fma(a, both(-1.f), both(1.f));
    }
}
template <bool LOGIT> __device__ __forceinline__ void decay_of(float2 raw, F2 &a, F2 &na) {
    if constexpr (LOGIT) {
        float g0, g1;
        asm("max.NaN.f32 %0, %1, %2;\n\tmin.NaN.f32 %0, %0, %3;" : "=&f"(g0) : "f"(raw.x), "f"(-88.5f), "f"(88.5f));
        asm("max.NaN.f32 %0, %1, %2;\n\tmin.NaN.f32 %0, %0, %3;" : "=&f"(g1) : "f"(raw.y), "f"(-88.5f), "f"(88.5f));
        const F2 g(g0, g1), c = both(-1.4426950408889634f), t = mul(g, c), off = fma(g, both(-1.9259630e-8f), fma(g, c, mul(t, both(-1.f))));
        F2 e(exp2_fast(t.x()), exp2_fast(t.y()));
        e = fma(mul(e, off), both(0.6931471805599453f), e);
        const F2 d = add(e, both(1.f)), r(rcp_fast(d.x()), rcp_fast(d.y()));
        a = mul(r, fma(mul(d, both(-1.f)), r, both(2.f)));
        const F2 up = mul(e, a), down = fma(a, both(-1.f), both(1.f));
        na = F2(g0 < 0.f ? down.x() : up.x(), g1 < 0.f ? down.y() : up.y());
    } else {
        a = F2(raw.x, raw.y);
        na = fma(a, both(-1.f), both(1.f));
    }
}

__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits for all but the last `N` groups of the thread's copies, then for its warp.
template <int N> __device__ __forceinline__ void copies_landed() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}
// Pairs between the segments of a stage: half-warps of 4-byte pairs would meet in the same banks.
template <typename XT, int S> __host__ __device__ constexpr int segment_pairs(int width) {
    return S * width + (sizeof(XT) == 2 && width == 16 ? 16 : 0);
}

// Where a thread stands: its pair of channels and its segment.
template <typename XT, bool WIDE, int S, int QT, bool CL> struct Place {
    using E = Elem<XT>;
    using One = typename E::One;
    using Pair = typename E::Pair;
    int q_all;                   // segments of the block, QT where that is fixed
    int cp, q, rank;             // own pair, own segment, block in the cluster
    int64_t m, b;                // first channel, its sample
    bool on, on2;                // the pair, its second channel
    int64_t sample;              // of the first of the warp's pairs of the segment
    bool one_sample;             // it is that of the others too
    int span, step;              // steps of the block, of a pass
    int64_t base;                // elements to the block's first channel
    uint32_t off, st;            // bytes to the thread's channels and segment, of a step
    // The 16-byte piece that the thread copies of every kPairs-th row: its first row (beyond every
    // segment where the piece lies beyond the last channel), bytes to it in memory and in a segment's slots.
    static constexpr int kPairs = 16 / sizeof(Pair);
    int piece_row;
    uint32_t piece_off, piece_slot;
    __device__ __forceinline__ int Q() const { return QT ? QT : q_all; }
    __device__ __forceinline__ int pairs() const { return QT ? 256 / (QT ? QT : 1) : 256 / q_all; }
    __device__ __forceinline__ explicit Place(const ScanArgs &P) {
        q_all = P.Q;
        const int width = pairs();
        cp = threadIdx.x % width;
        q = threadIdx.x / width;
        rank = CL ? blockIdx.x % P.CT : 0;
        const int64_t g0 = (int64_t)(CL ? blockIdx.x / P.CT : blockIdx.x) * width, g = g0 + cp;
        on = g < P.pairs;
        b = on ? g / P.PN : 0;
        const int64_t n = on ? 2 * (g % P.PN) : 0, b0 = g0 / P.PN, n0 = 2 * (g0 % P.PN);
        on2 = on && (WIDE || n + 1 < P.N);
        m = b * P.N + n;
        span = Q() * S;
        step = span * (CL ? P.CT : 1);
        base = b0 * P.sb + n0;
        st = (uint32_t)(P.st * sizeof(XT));
        const int lane = threadIdx.x & 31;
        sample = __shfl_sync(0xffffffffu, b, lane - lane % min(32, width));
        one_sample = __all_sync(0xffffffffu, !on || b == sample);
        off = on ? (uint32_t)(((b - b0) * P.sb + n - n0) * (int64_t)sizeof(XT)) + (uint32_t)(q * S) * st : 0;
        const int across = min(32, width) / kPairs, row = (cp & 31) / across;
        const int piece = (cp & ~31) + (cp & 31) % across * kPairs;
        const int64_t gp = g0 + piece;
        piece_row = gp < P.pairs ? row : INT32_MAX / 2;
        piece_off = gp < P.pairs ? (uint32_t)((((gp / P.PN) - b0) * P.sb + 2 * (gp % P.PN) - n0) * (int64_t)sizeof(XT)) +
                                       (uint32_t)(q * S + row) * st : 0;
        piece_slot = (uint32_t)((row * width + piece) * sizeof(Pair));
    }
    // Copies the rows of this thread's segment from `p` into `to`, S rows of `width` pairs; the
    // threads of a warp share the work where rows are WIDE (16-byte pieces), else each
    // copies its own pair.
    __device__ __forceinline__ void copy(Pair *to, const char *p, int left) const {
        const int width = pairs();
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
        if constexpr (WIDE) {
#pragma unroll
            for (int r = 0; r < S; r += kPairs)
                if (r < left - piece_row)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                                         dst + piece_slot + (uint32_t)(r * width * sizeof(Pair))),
                                     "l"(p + (piece_off + r * st)) : "memory");
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (on && s < left) {
                    const One *at = reinterpret_cast<const One *>(p + (off + s * st));
                    if constexpr (sizeof(One) == 4) {
                        const uint32_t d = dst + (uint32_t)((s * width + cp) * sizeof(Pair));
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(at) : "memory");
                        if (on2)
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d + 4), "l"(at + 1) : "memory");
                    } else {
                        to[s * width + cp] = E::pair(__ldcs(at), on2 ? __ldcs(at + 1) : One());
                    }
                }
        }
    }
    // Writes the rows of this thread's segment from `from`, where the threads of the warp have put
    // them, to `p`: the way of copy, back.
    __device__ __forceinline__ void write(char *p, const Pair *from, int left) const {
        const int width = pairs();
        if constexpr (WIDE) {
            const char *src = reinterpret_cast<const char *>(from) + piece_slot;
#pragma unroll
            for (int r = 0; r < S; r += kPairs)
                if (r < left - piece_row)
                    __stcs(reinterpret_cast<uint4 *>(p + (piece_off + r * st)),
                           *reinterpret_cast<const uint4 *>(src + r * width * sizeof(Pair)));
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (on && s < left) {
                    One *at = reinterpret_cast<One *>(p + (off + s * st));
                    const Pair w = from[s * width + cp];
                    __stcs(at, E::first(w));
                    if (on2) __stcs(at + 1, E::second(w));
                }
        }
    }
    // States of the pair, [B, N] float32.
    __device__ __forceinline__ F2 state(const float *p) const {
        return F2(on && p ? p[m] : 0.f, on2 && p ? p[m + 1] : 0.f);
    }
    __device__ __forceinline__ void put_state(float *p, F2 v) const {
        if (on) p[m] = v.x();
        if (on2) p[m + 1] = v.y();
    }
    // Start flags. Threads side by side whose pairs are of one sample read one flag each, for as
    // many passes at once as they reach (`ask`), a group of passes ahead of their use; `starts`
    // gives the S flags of the segment at t0. (One read a pass cost the forward of
    // 2048 steps of 65536 bfloat16 channels 28 us of 160: its way back is waited for with whatever else the warp reads.) By whole warps.
    __device__ __forceinline__ int group() const { return min(32, pairs()) / S; }
    // `hop`: steps from a pass to the next, negative where they run backwards.
    __device__ __forceinline__ uint32_t ask(const ScanArgs &P, int t0, int hop) const {
        const int l = (threadIdx.x & 31) % min(32, pairs()), t = t0 + l / S * hop + l % S;
        return P.starts && one_sample && t >= 0 && t < P.T ? P.starts[(int64_t)t * P.ft + sample * P.fb] : 0;
    }
    __device__ __forceinline__ uint32_t gather(uint32_t asked) const {
        const int lane = threadIdx.x & 31;
        return __ballot_sync(0xffffffffu, asked) >> (lane - lane % min(32, pairs()));
    }
    __device__ __forceinline__ uint32_t starts(const ScanArgs &P, int t0, uint32_t gathered, int pass) const {
        if (!P.starts) return 0;
        if (one_sample) return gathered >> pass % group() * S & ((1u << S) - 1);
        uint32_t f = 0;
        if (on)
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (t0 + s < P.T && P.starts[(int64_t)(t0 + s) * P.ft + b * P.fb]) f |= 1u << s;
        return f;
    }
};

template <typename XT, bool WIDE, int S, int QT, bool LOGIT, bool MIX, bool CL>
__global__ void __launch_bounds__(256, 2) scan_forward_kernel(const ScanArgs P) {
    using E = Elem<XT>;
    using Pair = typename E::Pair;
    constexpr int kStages = kForwardStages<XT>;
    pdl_begin();
    __shared__ ScanShared<CL> sh;
    const Place<XT, WIDE, S, QT, CL> me(P);
    const int width = me.pairs(), Q = me.Q();
    constexpr int MQ = QT ? QT : 8;                // most segments
    F2 carry = me.state(P.h0);                     // read by every block before any can write h_last over it
    enter_cluster<CL>(sh, P.CT, width);
    if (P.T == 0) {
        if (me.q == 0 && me.rank == 0 && P.last) me.put_state(P.last, carry);
        leave_cluster<CL>(sh);
        return;
    }
    const int64_t first = (me.base + (int64_t)(me.rank * me.span) * P.st) * (int64_t)sizeof(XT);
    const int64_t hop = (int64_t)me.step * P.st * (int64_t)sizeof(XT);
    const char *px = static_cast<const char *>(P.x) + first, *pg = static_cast<const char *>(P.gate) + first;
    char *ph = static_cast<char *>(P.h) + first;
    extern __shared__ __align__(16) unsigned char dynamic[];
    const int seg = segment_pairs<XT, S>(width), stage_pairs = 2 * Q * seg;
    Pair *slots = reinterpret_cast<Pair *>(dynamic) + me.q * seg;
    int t0 = me.rank * me.span + me.q * S;
    uint32_t asked = me.ask(P, t0, me.step), gathered = 0;
    // the rows of the pass that begins at step t for this thread
    auto fetch = [&](int stage, int t) {
        Pair *to = slots + stage * stage_pairs;
        me.copy(to, pg, P.T - t);
        me.copy(to + Q * seg, px, P.T - t);
        copies_issued();
        pg += hop;
        px += hop;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, t0 + i * me.step);
    int stage = 0;
    for (int pass = 0; (int64_t)pass * me.step < P.T; ++pass) {
        F2 a[S], u[S], A, B;
        if (pass % me.group() == 0) {
            gathered = me.gather(asked);
            asked = me.ask(P, t0 + me.group() * me.step, me.step);
        }
        const uint32_t cut = me.starts(P, t0, gathered, pass);
        const int t1 = t0, left = P.T - t0;       // steps of the sequence from this segment on
        // the usual segments: whole, without a start in any lane
        const bool plain = __all_sync(0xffffffffu, left >= S && !cut);
        copies_landed<kStages - 2>();
        Pair *xs = slots + stage * stage_pairs + Q * seg, *xr = xs + me.cp;
        const Pair *gr = xr - Q * seg;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            F2 na;
            decay_of<LOGIT>(gr[s * width], a[s], na);
            u[s] = E::unpack(xr[s * width]);
            if (MIX) u[s] = mul(u[s], na);
        }
        __syncwarp();                             // the stage before this one is free
        fetch(stage == 0 ? kStages - 1 : stage - 1, t0 + (kStages - 1) * me.step);
        if (++stage == kStages) stage = 0;
        if (plain) {
            A = a[0];
            B = u[0];
#pragma unroll
            for (int s = 1; s < S; ++s) {
                A = mul(A, a[s]);
                B = fma(a[s], B, u[s]);
            }
        } else {
            A = both(1.f);
            B = both(0.f);
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s < left) {
                    A = mul(A, a[s]);
                    B = cut >> s & 1 ? u[s] : fma(a[s], B, u[s]);
                }
        }
        t0 += me.step;
        int flag = cut ? kCut : 0;
        if (!LOGIT && !cut) flag = growth<S>(a, left, A);
        bool flags;
        F2 h = fold<CL, LOGIT, MQ>(sh, P.CT, me.q, me.cp, width, me.rank, pass, A, B, flag, carry, flags);
        if (P.saved && t1 && t1 < P.T && t1 % kInterval == 0)
            me.put_state(P.saved + (int64_t)(t1 / kInterval - 1) * P.M, h);
        if (plain) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                h = fma(a[s], h, u[s]);
                xr[s * width] = E::pack(h);
            }
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s < left) {
                    h = cut >> s & 1 ? u[s] : fma(a[s], h, u[s]);
                    xr[s * width] = E::pack(h);
                }
        }
        __syncwarp();
        me.write(ph, xs, left);
        ph += hop;
        if (P.last && left > 0 && left <= S) me.put_state(P.last, h);
        if (!CL && me.q == Q - 1) sh.carry[pass & 1][me.cp] = h;
    }
    leave_cluster<CL>(sh);
}

template <typename XT, bool WIDE, int S, int QT, bool LOGIT, bool MIX, bool CL>
__global__ void __launch_bounds__(256, 2) scan_backward_kernel(const ScanArgs P) {
    using E = Elem<XT>;
    using Pair = typename E::Pair;
    constexpr int kStages = kBackwardStages<XT>;
    pdl_begin();
    __shared__ ScanShared<CL> sh;
    __shared__ F2 ends[2][256];                              // B of the segments' forward maps
    const Place<XT, WIDE, S, QT, CL> me(P);
    const int width = me.pairs(), Q = me.Q();
    constexpr int MQ = QT ? QT : 8;                // most segments
    F2 carry = me.state(P.glast);                  // read by every block before any can write grad_h0 over it
    enter_cluster<CL>(sh, P.CT, width);
    if (P.T == 0) {
        if (me.q == 0 && me.rank == 0 && P.gh0) me.put_state(P.gh0, carry);
        leave_cluster<CL>(sh);
        return;
    }
    const int passes = (P.T - 1) / me.step + 1;
    int t0 = (passes - 1) * me.step + me.rank * me.span + me.q * S;
    const int64_t hop = (int64_t)me.step * P.st * (int64_t)sizeof(XT);
    const int64_t first = (me.base + (int64_t)(me.rank * me.span) * P.st) * (int64_t)sizeof(XT) + (passes - 1) * hop;
    const char *px = static_cast<const char *>(P.x) + first, *pg = static_cast<const char *>(P.gate) + first;
    const char *pl = static_cast<const char *>(P.gh) + first;
    char *pgx = static_cast<char *>(P.gx) + first, *pgg = static_cast<char *>(P.gg) + first;
    extern __shared__ __align__(16) unsigned char dynamic[];
    const int seg = segment_pairs<XT, S>(width), stage_pairs = 3 * Q * seg;
    Pair *slots = reinterpret_cast<Pair *>(dynamic) + me.q * seg;
    uint32_t asked = me.ask(P, t0, -me.step);   // one pass ahead: groups of passes were slower here (251 -> 327 us)
    // h before the block's first step of the pass whose segment begins at t
    auto begin = [&](int t) {
        const int tb = t - me.q * S;                         // a multiple of the interval, or 0
        return me.state(tb > 0 && tb < P.T ? P.saved + (int64_t)(tb / kInterval - 1) * P.M : tb == 0 ? P.h0 : nullptr);
    };
    F2 start = begin(t0);
    auto fetch = [&](int stage, int t) {
        if (t >= 0) {
            Pair *to = slots + stage * stage_pairs;
            me.copy(to, pg, P.T - t);
            me.copy(to + Q * seg, px, P.T - t);
            me.copy(to + 2 * Q * seg, pl, P.T - t);
        }
        copies_issued();
        pg -= hop;
        px -= hop;
        pl -= hop;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, t0 - i * me.step);
    int stage = 0;
    for (int pass = 0; pass < passes; ++pass) {
        F2 a[S], na[S], A = both(1.f), B = both(0.f), L = both(0.f), h = start;
        const uint32_t cut = me.starts(P, t0, me.gather(asked), 0);
        const int t1 = t0, left = P.T - t0;
        const bool plain = __all_sync(0xffffffffu, left >= S && !cut);
        copies_landed<kStages - 2>();
        Pair *gs = slots + stage * stage_pairs, *xs = gs + Q * seg, *gr = gs + me.cp, *xr = xs + me.cp;
        const Pair *lr = xr + Q * seg;
        auto gh_of = [&](int s) { return E::unpack(lr[s * width]); };
        auto x_of = [&](int s) { return E::unpack(xr[s * width]); };
#pragma unroll
        for (int s = 0; s < S; ++s) decay_of<LOGIT>(gr[s * width], a[s], na[s]);
        // what the state takes up in step s
        auto input = [&](int s) {
            const F2 u = x_of(s);
            return MIX ? mul(u, na[s]) : u;
        };
        if (plain) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                A = mul(A, a[s]);
                B = fma(a[s], B, input(s));
            }
#pragma unroll
            for (int s = S - 1; s >= 0; --s) L = mul(a[s], add(gh_of(s), L));
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s < left) {
                    A = mul(A, a[s]);
                    B = cut >> s & 1 ? input(s) : fma(a[s], B, input(s));
                }
#pragma unroll
            for (int s = S - 1; s >= 0; --s)
                if (s < left) L = cut >> s & 1 ? both(0.f) : mul(a[s], add(gh_of(s), L));
        }
        // the stage read in the pass before is free; its readers have passed copies_landed
        fetch(stage == 0 ? kStages - 1 : stage - 1, t0 - (kStages - 1) * me.step);
        if (++stage == kStages) stage = 0;
        t0 -= me.step;
        asked = me.ask(P, t0, -me.step);
        start = begin(t0);
        const int buf = pass & 1, from_end = Q - 1 - me.q;
        ends[buf][me.q * width + me.cp] = B;
        int flag = cut ? kCut : 0;
        if (!LOGIT && !cut) flag = growth<S>(a, left, A);
        bool flags;
        F2 mu = fold<CL, LOGIT, MQ>(sh, P.CT, from_end, me.cp, width, CL ? P.CT - 1 - me.rank : 0, pass, A, L, flag, carry, flags);
        // the forward maps have the same products of decays
        auto map = [&](int i) { return Map{sh.map[buf][(Q - 1 - i) * width + me.cp].A, ends[buf][i * width + me.cp]}; };
        auto flag_of = [&](int i) { return sh.flag[buf][(Q - 1 - i) * width + me.cp]; };
        h = flags ? fold_before<LOGIT, MQ, true>(me.q, h, map, flag_of) : fold_before<LOGIT, MQ, false>(me.q, h, map, flag_of);
        F2 before[S];
        // gradients of step s, from the state before it and mu after it
        auto gradients = [&](int s, F2 ga) {
            const F2 lam = add(gh_of(s), mu);
            if (MIX) ga = fma(x_of(s), both(-1.f), ga);
            ga = mul(ga, lam);
            if (LOGIT) ga = mul(ga, mul(a[s], na[s]));
            xr[s * width] = E::pack(MIX ? mul(lam, na[s]) : lam);
            gr[s * width] = E::pack(ga);
            mu = mul(a[s], lam);
        };
        if (plain) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                before[s] = h;
                if (s + 1 < S) h = fma(a[s], h, input(s));
            }
#pragma unroll
            for (int s = S - 1; s >= 0; --s) gradients(s, before[s]);
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (s < left) {
                    const bool c = cut >> s & 1;
                    before[s] = c ? both(0.f) : h;
                    h = c ? input(s) : fma(a[s], h, input(s));
                }
#pragma unroll
            for (int s = S - 1; s >= 0; --s)
                if (s < left) {
                    gradients(s, before[s]);
                    if (cut >> s & 1) mu = both(0.f);
                }
        }
        __syncwarp();
        me.write(pgx, xs, left);
        me.write(pgg, gs, left);
        pgx -= hop;
        pgg -= hop;
        if (t1 == 0 && P.gh0) me.put_state(P.gh0, mu);
        if (!CL && me.q == 0) sh.carry[buf][me.cp] = mu;
    }
    leave_cluster<CL>(sh);
}

// Step by step, one thread for a channel: rows so far apart that a block's 32-bit offsets
// cannot reach them (millions of channels, which fill the card without a split of time).
template <typename XT, bool LOGIT, bool MIX>
__global__ void __launch_bounds__(128) scan_forward_far_kernel(const ScanArgs P) {
    using E = Elem<XT>;
    using One = typename E::One;
    pdl_begin();
    const int64_t m = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (m >= P.M) return;
    const int64_t b = m / P.N, off = b * P.sb + m % P.N;
    float v = P.h0 ? P.h0[m] : 0.f;
    for (int t = 0; t < P.T; ++t) {
        const int64_t at = off + t * P.st;
        F2 a, na;
        decay_of<LOGIT>(E::pair(__ldcs(static_cast<const One *>(P.gate) + at), One()), a, na);
        float u = E::unpack(E::pair(__ldcs(static_cast<const One *>(P.x) + at), One())).x();
        if (MIX) u *= na.x();
        v = P.starts && P.starts[t * P.ft + b * P.fb] ? u : fmaf(a.x(), v, u);
        __stcs(static_cast<One *>(P.h) + at, E::first(E::pack(F2(v, 0.f))));
        if (P.saved && (t + 1) % kInterval == 0 && t + 1 < P.T) P.saved[(int64_t)(t / kInterval) * P.M + m] = v;
    }
    if (P.last) P.last[m] = v;
}

template <typename XT, bool LOGIT, bool MIX>
__global__ void __launch_bounds__(128) scan_backward_far_kernel(const ScanArgs P) {
    using E = Elem<XT>;
    using One = typename E::One;
    pdl_begin();
    const int64_t m = (int64_t)blockIdx.x * 128 + threadIdx.x;
    if (m >= P.M) return;
    const int64_t b = m / P.N, off = b * P.sb + m % P.N;
    auto value = [](const void *p, int64_t at) { return E::unpack(E::pair(static_cast<const One *>(p)[at], One())).x(); };
    float before[kInterval];                                 // h[t-1] of the interval's steps
    float mu = P.glast ? P.glast[m] : 0.f;
    for (int c = (P.T + kInterval - 1) / kInterval - 1; c >= 0; --c) {
        const int t0 = c * kInterval, t1 = min(P.T, t0 + kInterval);
        float v = c ? P.saved[(int64_t)(c - 1) * P.M + m] : P.h0 ? P.h0[m] : 0.f;
        for (int t = t0; t < t1; ++t) {
            const int64_t at = off + t * P.st;
            F2 a, na;
            decay_of<LOGIT>(E::pair(static_cast<const One *>(P.gate)[at], One()), a, na);
            const float x = value(P.x, at), u = MIX ? na.x() * x : x;
            before[t - t0] = v;
            v = P.starts && P.starts[t * P.ft + b * P.fb] ? u : fmaf(a.x(), v, u);
        }
        for (int t = t1 - 1; t >= t0; --t) {
            const int64_t at = off + t * P.st;
            F2 a, na;
            decay_of<LOGIT>(E::pair(static_cast<const One *>(P.gate)[at], One()), a, na);
            const float x = value(P.x, at);
            const bool start = P.starts && P.starts[t * P.ft + b * P.fb];
            const float lam = value(P.gh, at) + mu, hp = start ? 0.f : before[t - t0];
            const float ga = lam * (MIX ? hp - x : hp);
            __stcs(static_cast<One *>(P.gx) + at, E::first(E::pack(F2(MIX ? lam * na.x() : lam, 0.f))));
            __stcs(static_cast<One *>(P.gg) + at, E::first(E::pack(F2(LOGIT ? ga * (a.x() * na.x()) : ga, 0.f))));
            mu = start ? 0.f : a.x() * lam;
        }
    }
    if (P.gh0) P.gh0[m] = mu;
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
// Blocks of a call that takes clusters: all of them resident, also where a cluster of 8 does not
// fill its GPC.
constexpr int kMostClustered = 256;

template <typename XT, bool WIDE, bool LOGIT, bool MIX, bool FWD>
cudaError_t launch(ScanArgs a, cudaStream_t s) {
    // Steps of a segment: 8, and 4 in the float32 backward, whose segments of 8 would leave one
    // block an SM (a layer of T = 512, 16 x 4096: 172 us against 191).
    constexpr int S = sizeof(XT) == 4 && !FWD ? 4 : 8;
    constexpr int kFullQ = kInterval / S;      // segments that make an interval
    constexpr int W = 16;                      // most segments of a block
    a.PN = (a.N + 1) / 2;
    a.pairs = a.M / a.N * a.PN;
    // Time: as many segments as the steps fill, up to an interval; twice that, and then the
    // blocks of a cluster, while the channels alone leave SMs without one.
    a.Q = 1;
    while (a.Q < kFullQ && a.Q * S < a.T) a.Q *= 2;
    auto groups = [&] { return (a.pairs + 256 / a.Q - 1) / (256 / a.Q); };
    if (W > kFullQ && a.Q == kFullQ && a.T > a.Q * S && groups() < kBusy) a.Q *= 2;
    a.CT = 1;
    while (a.CT < 8 && groups() * a.CT * 2 <= kMostClustered && a.T > a.Q * S * a.CT) a.CT *= 2;
    // the farthest offset in a block: its samples apart (none where they are a block's multiple
    // of pairs), its steps apart
    const int width = 256 / a.Q;
    const int64_t reach = (a.PN % width ? ((width - 1) / a.PN + 1) * a.sb : 0) + a.N + (int64_t)a.Q * S * a.st;
    if (reach * (int64_t)sizeof(XT) > UINT32_MAX) {
        const unsigned blocks = (unsigned)((a.M + 127) / 128);
        if constexpr (FWD) return seq_launch(scan_forward_far_kernel<XT, LOGIT, MIX>, dim3(blocks), 128, 0, s, 1, a);
        else return seq_launch(scan_backward_far_kernel<XT, LOGIT, MIX>, dim3(blocks), 128, 0, s, 1, a);
    }
    const size_t smem = (size_t)(FWD ? 2 * kForwardStages<XT> : 3 * kBackwardStages<XT>) * a.Q *
                        segment_pairs<XT, S>(256 / a.Q) * sizeof(typename Elem<XT>::Pair);
    auto start = [&](auto kernel) {
        cudaError_t e = smem <= 16384 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        return seq_launch(kernel, dim3((unsigned)(groups() * a.CT)), 256, smem, s, a.CT, a);
    };
    // QT: the segments of a block where the steps fill an interval, 0 for shorter sequences
    if constexpr (FWD)
        return a.CT > 1        ? start(scan_forward_kernel<XT, WIDE, S, W, LOGIT, MIX, true>)
               : a.Q < kFullQ  ? start(scan_forward_kernel<XT, WIDE, S, 0, LOGIT, MIX, false>)
               : a.Q == kFullQ ? start(scan_forward_kernel<XT, WIDE, S, kFullQ, LOGIT, MIX, false>)
                               : start(scan_forward_kernel<XT, WIDE, S, W, LOGIT, MIX, false>);
    else
        return a.CT > 1        ? start(scan_backward_kernel<XT, WIDE, S, W, LOGIT, MIX, true>)
               : a.Q < kFullQ  ? start(scan_backward_kernel<XT, WIDE, S, 0, LOGIT, MIX, false>)
               : a.Q == kFullQ ? start(scan_backward_kernel<XT, WIDE, S, kFullQ, LOGIT, MIX, false>)
                               : start(scan_backward_kernel<XT, WIDE, S, W, LOGIT, MIX, false>);
}

// Rows are copied 16 bytes at a time where they are aligned to 16 bytes in every tensor.
template <typename XT, bool LOGIT, bool MIX>
cudaError_t launch_form(bool forward, const ScanArgs &a, cudaStream_t s) {
    const bool wide = a.N * sizeof(XT) % 16 == 0 && seq_aligned(a.x, 16) && seq_aligned(a.gate, 16) &&
                      seq_aligned(a.h, 16) && seq_aligned(a.gh, 16) && seq_aligned(a.gx, 16) && seq_aligned(a.gg, 16);
    if (forward) return wide ? launch<XT, true, LOGIT, MIX, true>(a, s) : launch<XT, false, LOGIT, MIX, true>(a, s);
    return wide ? launch<XT, true, LOGIT, MIX, false>(a, s) : launch<XT, false, LOGIT, MIX, false>(a, s);
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
