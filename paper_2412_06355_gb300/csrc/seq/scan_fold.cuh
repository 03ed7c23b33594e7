// The maps of a pass of the gated scan: folded over the state within a block through shared memory,
// between the blocks of a cluster by asynchronous stores.
#pragma once

#include <cooperative_groups.h>
#include <stdint.h>

#include "pairs.cuh"
#include "waits.cuh"

namespace dendsn {

// A h + B of a segment's map over a state, B alone where the segment has a start.
__device__ __forceinline__ F2 map_over(F2 A, F2 B, bool cut, F2 h) {
    const F2 r = fma(A, h, B);
    return cut ? B : r;
}
// A product of decays, kept finite: a state of zero stays zero under decays above 1 whose
// product overflows. (Where a decay is NaN, so is the segment's end.)
template <bool LOGIT> __device__ __forceinline__ F2 finite(F2 A) {
    constexpr float top = 3.402823466e38f;
    if constexpr (LOGIT) return A;
    else return F2(fminf(fmaxf(A.x(), -top), top), fminf(fmaxf(A.y(), -top), top));
}
struct alignas(16) Map {
    F2 A, B;
};
__device__ __forceinline__ F2 over(const Map &m, bool cut, F2 h) { return map_over(m.A, m.B, cut, h); }

// Maps of the segments, in two buffers of alternating passes.
template <bool CL> struct ScanShared {
    Map map[2][256];                             // [segment in the order of the fold][pair]
    F2 carry[2][256];                            // the state at the end of a pass
    Map block[2][CL ? 8 : 1][CL ? 32 : 1];       // maps of the cluster's blocks
    int32_t block_cut[2][CL ? 8 : 1][CL ? 32 : 1];
    uint64_t arrived[2];                         // barriers that count their bytes
    bool cut[2][256];
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
    __device__ __forceinline__ void send(int buf, int mine, int cp, const Map &m, bool cut) const {
        for (int r = 0; r < blocks; ++r) {
            uint32_t to, flag, bar;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(addr(&sh.block[buf][mine][cp])), "r"(r));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(flag) : "r"(addr(&sh.block_cut[buf][mine][cp])), "r"(r));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(addr(&sh.arrived[buf])), "r"(r));
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                         ::"r"(to), "f"(m.A.x()), "f"(m.A.y()), "f"(m.B.x()), "f"(m.B.y()), "r"(bar) : "memory");
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(flag),
                         "r"((int)cut), "r"(bar) : "memory");
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

// Folds the segment maps over the state before the pass; returns the state before this
// thread's segment, which is number `me` of Q in the order of the fold, and whether any segment
// of the block has a start. One barrier a pass: the maps have two buffers, and the last segment
// leaves the state behind in sh.carry.
//
// A block whose maps do not come takes NaN for the state before it from then on (starts within the
// block still begin anew), waits no more and sends no more: its buffers may hold maps of another
// pass, and so would those of blocks that still read what it sent.
template <bool CL, bool LOGIT, int MQ>
__device__ __forceinline__ F2 fold(ScanShared<CL> &sh, int CT, int me, int cp, int width, int mine,
                                   int pass, F2 A, F2 B, bool cut, F2 &carry, bool &cuts) {
    const int buf = pass & 1;
    sh.map[buf][me * width + cp] = Map{finite<LOGIT>(A), B};
    sh.cut[buf][me * width + cp] = cut;
    F2 in;
    if constexpr (!CL) {
        cuts = __syncthreads_or(cut);
        in = pass ? sh.carry[buf ^ 1][cp] : carry;
        // unrolled, so that the maps are read together and only the products wait on one another
        if (cuts) {
#pragma unroll
            for (int i = 0; i < MQ - 1; ++i)
                if (i < me) in = over(sh.map[buf][i * width + cp], sh.cut[buf][i * width + cp], in);
        } else {
#pragma unroll
            for (int i = 0; i < MQ - 1; ++i)
                if (i < me) in = over(sh.map[buf][i * width + cp], false, in);
        }
    } else {
        const Exchange<CL> ex{sh, CT, width};
        cuts = __syncthreads_or(cut);
        const bool lost = sh.lost;
        if (me == 0) {                           // the block's map, handed to every block
            F2 a = both(1.f), b = both(0.f);
            bool c = false;
#pragma unroll
            for (int i = 0; i < MQ; ++i) {
                const Map m = sh.map[buf][i * width + cp];
                const bool ci = cuts && sh.cut[buf][i * width + cp];
                b = over(m, ci, b);
                a = finite<LOGIT>(mul(a, m.A));
                c |= ci;
            }
            if (!lost) ex.send(buf, mine, cp, Map{a, b}, c);
        }
        const bool here = ex.wait(buf, pass >> 1 & 1, lost);
        if (threadIdx.x == 0 && here) ex.expect(buf);
        in = carry;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < CT) {
                carry = over(sh.block[buf][i][cp], sh.block_cut[buf][i][cp], carry);
                if (i + 1 == mine) in = carry;
            }
        if (!here) {
            sh.lost = 1;
            in = carry = both(__int_as_float(0x7fffffff));
        }
        if (cuts) {
            for (int i = 0; i < me; ++i) in = over(sh.map[buf][i * width + cp], sh.cut[buf][i * width + cp], in);
        } else {
#pragma unroll
            for (int i = 0; i < MQ - 1; ++i)
                if (i < me) in = over(sh.map[buf][i * width + cp], false, in);
        }
    }
    return in;
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
