// The maps of a pass of the gated scan: folded over the state within a block through shared memory,
// between the blocks of a cluster by asynchronous stores.
#pragma once

#include <cooperative_groups.h>
#include <stdint.h>

#include "pairs.cuh"
#include "waits.cuh"

namespace dendsn {

// The map h -> A h + B of a segment or of a block's segments, with a flag:
//   kCut   a sequence starts within: the map is constant, B
//   else   the exponents of the two channels (0: A as it is). Where decays above 1 are multiplied,
//          the product may leave float32 although the states do not (growth that falls back, or from
//          a tiny state): that channel's A is then a mantissa, to be scaled by 2^exponent (within
//          1000: a state that is not zero leaves float32 long before).
// Each channel by itself: what a channel gets does not depend on the one beside it.
struct alignas(16) Map {
    F2 A, B;
};
constexpr int kCut = 1, kWild = ~1;

__device__ __forceinline__ F2 over(const Map &m, bool cut, F2 h) {
    const F2 r = fma(m.A, h, m.B);
    return cut ? m.B : r;
}
__device__ __forceinline__ int wild_field(int flag, int channel) { return flag >> (channel ? 12 : 1) & 2047; }
__device__ __forceinline__ double power_of_2(int e) { return __hiloint2double((e + 1023) << 20, 0); }
__device__ __forceinline__ double wild_product(float A, int field) {
    return field ? (double)A * power_of_2(field - 1024) : (double)A;
}
// over() with any flag.
__device__ __forceinline__ float over_wild(float A, float B, int field, float h) {
    return field ? (float)::fma(wild_product(A, field), (double)h, (double)B) : fmaf(A, h, B);
}
__device__ __forceinline__ F2 over_wild(const Map &m, int flag, F2 h) {
    if (flag & kCut) return m.B;
    return F2(over_wild(m.A.x(), m.B.x(), wild_field(flag, 0), h.x()), over_wild(m.A.y(), m.B.y(), wild_field(flag, 1), h.y()));
}
// Mantissa and field of a product.
__device__ __forceinline__ int split_wild(double v, float &A) {
    int e = (__double2hiint(v) >> 20 & 2047) - 1023;
    if (e > 1000 && e <= 1023) e = 1000;                      // finite
    const bool as_is = e < -1000 || e > 1000;                 // next to zero; infinite or NaN
    A = (float)(as_is ? v : v * power_of_2(-e));
    return (as_is ? 0 : e) + 1024;
}
// The flag of a segment of `left` steps (or S) without a start; where a channel has a decay above 1,
// its product of decays in A becomes the mantissa.
template <int S> __device__ __forceinline__ int growth(const F2 (&a)[S], int left, F2 &A) {
    float mx = 0.f, my = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (s < left) {
            mx = fmaxf(mx, fabsf(a[s].x()));
            my = fmaxf(my, fabsf(a[s].y()));
        }
    if (!(fmaxf(mx, my) > 1.f)) return 0;
    double x = 1., y = 1.;
#pragma unroll
    for (int s = 0; s < S; ++s)
        if (s < left) {
            x *= (double)a[s].x();
            y *= (double)a[s].y();
        }
    float ax = A.x(), ay = A.y();
    int flag = 0;
    if (mx > 1.f) flag |= split_wild(x, ax) << 1;
    if (my > 1.f) flag |= split_wild(y, ay) << 12;
    A = F2(ax, ay);
    return flag;
}

// Maps of the segments, in two buffers of alternating passes.
template <bool CL> struct ScanShared {
    Map map[2][256];                             // [segment in the order of the fold][pair]
    F2 carry[2][256];                            // the state at the end of a pass
    Map block[2][CL ? 8 : 1][CL ? 32 : 1];       // maps of the cluster's blocks
    int32_t block_flag[2][CL ? 8 : 1][CL ? 32 : 1];
    uint64_t arrived[2];                         // barriers that count their bytes
    int32_t flag[2][256];
    int32_t lost;                                // a pass's maps did not come
};

// Blocks of a cluster hand one another their maps by asynchronous stores, which count
// themselves in on the receiver's barrier: a cluster-wide barrier would also wait for every
// write of h on its way to memory (16384 steps of 1024 float32 channels: 71 us with one, 51 without).
// Buffers need no other guard: a block sends pass k + 2 after it has every map of pass k + 1,
// and a block sends those after its threads have read pass k.
template <bool CL> struct Exchange {
    ScanShared<CL> &sh;
    int blocks;                                  // of the cluster
    int width;
    __device__ __forceinline__ static uint32_t addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
    __device__ __forceinline__ void expect(int buf) const {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(addr(&sh.arrived[buf])),
                     "r"(blocks * width * 20) : "memory");
    }
    __device__ __forceinline__ void begin() const {
        if (threadIdx.x == 0) {
            for (int i = 0; i < 2; ++i)
                asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(addr(&sh.arrived[i])) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            expect(0);
            expect(1);
            sh.lost = 0;
        }
        cooperative_groups::this_cluster().sync();
    }
    __device__ __forceinline__ void send(int buf, int mine, int cp, const Map &m, int word) const {
        for (int r = 0; r < blocks; ++r) {
            uint32_t to, flag, bar;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(addr(&sh.block[buf][mine][cp])), "r"(r));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(flag) : "r"(addr(&sh.block_flag[buf][mine][cp])), "r"(r));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(addr(&sh.arrived[buf])), "r"(r));
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                         ::"r"(to), "f"(m.A.x()), "f"(m.A.y()), "f"(m.B.x()), "f"(m.B.y()), "r"(bar) : "memory");
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(flag),
                         "r"(word), "r"(bar) : "memory");
        }
    }
    __device__ __forceinline__ bool lost() const { return *const_cast<volatile int32_t *>(&sh.lost) != 0; }
    // Waits for the maps of a pass; false where they did not come within about a second, or where
    // another thread of the block has found that; at once where they are not to be waited for.
    __device__ __forceinline__ bool wait(int buf, uint32_t parity, bool skip) const {
        uint64_t began = 0;
        for (uint32_t i = 0; !skip; ++i) {
            uint32_t done;
            asm volatile("{\n\t.reg .pred p;\n\t"
                         "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                         "selp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done) : "r"(addr(&sh.arrived[buf])), "r"(parity) : "memory");
            if (done) return true;
            if (i % 64 == 63) {
                const uint64_t now = now_ns();
                if (lost()) return false;
                if (!began) began = now;
                else if (now - began > 1000000000ull) return false;
            }
        }
        return false;
    }
};

// The segments before number `me`, one after the other, over a state. FLAGS: some segment of the
// block has one. Unrolled, so that the maps are read together and only the products wait on one another;
// flags of growth, which LOGIT decays never have, are found on the way and taken in a second round.
template <bool LOGIT, int MQ, bool FLAGS, typename M, typename F>
__device__ __forceinline__ F2 fold_before(int me, F2 h, M map, F flag) {
    const F2 before = h;
    int any = 0;
#pragma unroll
    for (int i = 0; i < MQ - 1; ++i)
        if (i < me) {
            const int f = FLAGS ? flag(i) : 0;
            if (FLAGS && !LOGIT) any |= f;
            h = over(map(i), f & kCut, h);
        }
    if (FLAGS && !LOGIT && any & kWild) {
        h = before;
#pragma unroll 1
        for (int i = 0; i < me; ++i) h = over_wild(map(i), flag(i), h);
    }
    return h;
}

// Folds the segment maps over the state before the pass; returns the state before this
// thread's segment, which is number `me` of Q in the order of the fold, and whether any segment
// of the block has a flag. One barrier a pass: the maps have two buffers, and the last segment
// leaves the state behind in sh.carry.
//
// A block whose maps do not come takes NaN for the state before it from then on (starts within the
// block still begin anew), waits no more and sends no more: its buffers may hold maps of another
// pass, and so would those of blocks that still read what it sent.
template <bool CL, bool LOGIT, int MQ>
__device__ __forceinline__ F2 fold(ScanShared<CL> &sh, int CT, int me, int cp, int width, int mine,
                                   int pass, F2 A, F2 B, int flag, F2 &carry, bool &flags) {
    const int buf = pass & 1;
    sh.map[buf][me * width + cp] = Map{A, B};
    sh.flag[buf][me * width + cp] = flag;
    auto map = [&](int i) { return sh.map[buf][i * width + cp]; };
    auto flag_of = [&](int i) { return sh.flag[buf][i * width + cp]; };
    flags = __syncthreads_or(flag);
    F2 in;
    if constexpr (!CL) {
        in = pass ? sh.carry[buf ^ 1][cp] : carry;
    } else {
        const Exchange<CL> ex{sh, CT, width};
        const bool lost = sh.lost;
        if (me == 0) {                           // the block's map, handed to every block
            F2 a = both(1.f), b = both(0.f);
            int all = 0;
#pragma unroll
            for (int i = 0; i < MQ; ++i) {
                const Map m = map(i);
                const int f = flags ? flag_of(i) : 0;
                b = over(m, f & kCut, b);
                a = mul(a, m.A);
                all |= f;
            }
            if (!LOGIT && all & kWild) {
                constexpr double most = 1.0715086071862673e301;        // 2^1000
                double x = 1., y = 1.;
                b = both(0.f);
#pragma unroll 1
                for (int i = 0; i < MQ; ++i) {
                    const Map m = map(i);
                    const int f = flag_of(i);
                    b = over_wild(m, f, b);
                    x = ::fmin(::fmax(x * wild_product(m.A.x(), wild_field(f, 0)), -most), most);
                    y = ::fmin(::fmax(y * wild_product(m.A.y(), wild_field(f, 1)), -most), most);
                }
                float ax = a.x(), ay = a.y();
                const int fx = wild_field(all, 0) ? split_wild(x, ax) : 0, fy = wild_field(all, 1) ? split_wild(y, ay) : 0;
                a = F2(ax, ay);
                all = (all & kCut) | fx << 1 | fy << 12;
            }
            if (all & kCut) all = kCut;
            if (!lost) ex.send(buf, mine, cp, Map{a, b}, all);
        }
        const bool here = ex.wait(buf, pass >> 1 & 1, lost);
        if (threadIdx.x == 0 && here) ex.expect(buf);
        const F2 before = carry;
        int any = 0;
        in = carry;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < CT) {
                const int f = sh.block_flag[buf][i][cp];
                carry = over(sh.block[buf][i][cp], f & kCut, carry);
                any |= f;
                if (i + 1 == mine) in = carry;
            }
        if (!LOGIT && any & kWild) {
            in = carry = before;
#pragma unroll 1
            for (int i = 0; i < CT; ++i) {
                carry = over_wild(sh.block[buf][i][cp], sh.block_flag[buf][i][cp], carry);
                if (i + 1 == mine) in = carry;
            }
        }
        if (!here) {
            sh.lost = 1;
            in = carry = both(__int_as_float(0x7fffffff));
        }
    }
    return flags ? fold_before<LOGIT, MQ, true>(me, in, map, flag_of) : fold_before<LOGIT, MQ, false>(me, in, map, flag_of);
}

template <bool CL> __device__ __forceinline__ void enter_cluster(ScanShared<CL> &sh, int CT, int width) {
    if constexpr (CL) Exchange<CL>{sh, CT, width}.begin();
}
template <bool CL> __device__ __forceinline__ void leave_cluster(ScanShared<CL> &sh) {
    if constexpr (CL) {
        cooperative_groups::this_cluster().sync();   // no block sends any more
        // a block that has every map has seen its stores land; one that lost some lets those on
        // their way land first
        if (Exchange<CL>{sh, 0, 0}.lost()) let_land();
    }
}

}  // namespace dendsn
