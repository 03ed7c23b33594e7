// tcgen05 in a block of its own (cta_group::1): products of 128 rows whose left factor lies in tensor memory, or in
// shared memory, and whose right factor lies in shared memory as 8 x 8 blocks (fragments.cuh) without a swizzle.
#pragma once

#include "fragments.cuh"

namespace dendsn {
namespace tc {

__device__ __forceinline__ void tmem_alloc_one(uint32_t dst, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_one(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
// Left factor in tensor memory: a lane a row, a column two neighbours of the summed index.
__device__ __forceinline__ void mma_lanes(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
                 "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_tiles(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"((uint32_t)add) : "memory");
}
// Arrives at `bar` once the products this thread issued so far are done.
__device__ __forceinline__ void commit_one(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A tile of 8 x 8 blocks as an operand. `summed`: bytes between blocks along the summed index; `other`: along the other
// one. Which of the two runs along a block's 16-byte rows is the instruction's to say (product_of). `further` bytes on
// in the tile (addresses stay below 2^18, so the low word's upper half is not touched).
struct Blocks {
    uint32_t low, high;
    __device__ __forceinline__ Blocks(uint32_t addr, uint32_t summed, uint32_t other)
        : low(addr >> 4 | (summed >> 4) << 16), high(other >> 4 | 1u << 14) {}
    __device__ __forceinline__ uint64_t at(uint32_t further) const { return (uint64_t)high << 32 | (low + (further >> 4)); }
};
// 8 columns of this warp's 32 lanes; tmem_stored waits for all of them.
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void tmem_put(uint32_t addr, const float (&v)[16]) {
    uint32_t q[2][8];
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i / 8][i % 8] = __float_as_uint(v[i]);
    tmem_store(addr, q[0]);
    tmem_store(addr + 8, q[1]);
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 columns; one statement loads and waits.
__device__ __forceinline__ void tmem_load(float (&v)[16], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(addr) : "memory");
}

// A wait of a whole warp, in turn with those before it (`ok`): true for all its lanes or for none. Each lane looks at
// the clock by itself, so where a wait runs out lanes may disagree; what all of them have to execute together
// (elected below names all 32) stands behind a value that is one for the warp.
__device__ __forceinline__ bool warp_wait(bool ok, uint32_t bar, uint32_t parity) {
    ok = ok && bar_wait(bar, parity);
    return __all_sync(0xffffffffu, ok);
}
// One lane of a whole warp, in a way that leaves the compiler's uniform registers usable.
__device__ __forceinline__ bool elected() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

// Products of NA terms in tensor memory (STEPS blocks of 16 summed places, 8 columns each) and NB terms in shared
// memory, those whose terms' numbers add up to less than KEEP, the smallest first. TURNED: the right factor's rows
// run along the summed index, else along the other one. WIDTH: blocks of a row. TRI: of a lower triangle's rows only
// those from the step on (1), of its columns only those up to the step (2).
template <int NA, int NB, int KEEP, int STEPS, int N, int WIDTH, bool TURNED, int TRI>
__device__ __forceinline__ void issue(uint32_t d, uint32_t a, uint32_t aterm, uint32_t b, uint32_t bterm) {
    const Blocks tile = TURNED ? Blocks(b, WIDTH * kCell, kCell) : Blocks(b, kCell, WIDTH * kCell);
    bool add = false;
#pragma unroll
    for (int sum = KEEP - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = sum - i;
            if (j < 0 || j >= NB) continue;
#pragma unroll
            for (int n = 0; n < STEPS; ++n) {
                const int s = TRI == 2 ? STEPS - 1 - n : n;
                const int from = TRI == 1 ? 16 * s : 0, count = TRI == 1 ? N - 16 * s : TRI == 2 ? 16 * (s + 1) : N;
                mma_lanes(d + from, a + i * aterm + 8 * s, tile.at(j * bterm + (TURNED ? 2 * s * WIDTH : from / 8 * WIDTH + 2 * s) * kCell),
                          product_of(128, count, false, TURNED), add);
                add = true;
            }
        }
}
// The same of a left factor in shared memory whose rows run along the summed index (AW blocks a row), for `steps` blocks
// of 16 summed places, of the products whose terms' numbers add up to FROM and less than KEEP. add: onto what is there.
template <int NA, int NB, int FROM, int KEEP, int AW, int WIDTH, bool TURNED, int TRI>
__device__ __forceinline__ void issue_tiles(uint32_t d, uint32_t a, uint32_t aterm, uint32_t b, uint32_t bterm, int steps, bool add) {
    const Blocks left(a, AW * kCell, kCell), right = TURNED ? Blocks(b, WIDTH * kCell, kCell) : Blocks(b, kCell, WIDTH * kCell);
#pragma unroll
    for (int sum = KEEP - 1; sum >= FROM; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = sum - i;
            if (j < 0 || j >= NB) continue;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int s = TRI == 2 ? 3 - n : n;
                if (!TRI && s >= steps) continue;
                const int from = TRI == 1 ? 16 * s : 0, count = TRI == 1 ? 64 - 16 * s : TRI == 2 ? 16 * (s + 1) : 64;
                mma_tiles(d + from, left.at(i * aterm + 2 * s * AW * kCell), right.at(j * bterm + (TURNED ? 2 * s * WIDTH : from / 8 * WIDTH + 2 * s) * kCell),
                          product_of(128, count, true, TURNED), add);
                add = true;
            }
        }
}

// What threads wrote to shared memory, before products read it.
__device__ __forceinline__ void fence_tiles() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

}  // namespace tc
}  // namespace dendsn
