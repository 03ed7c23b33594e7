// Inline PTX of the tensor-core path: mbarriers, tensor copies, tcgen05 on a pair of blocks.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "waits.cuh"

namespace dendsn {
namespace tc {

__device__ __forceinline__ uint32_t smem_addr(const void *p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
// The address in block `rank` of the cluster of what lies at `addr` in this block.
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ------------------------------------------------------------------ mbarriers
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One arrival at a barrier of any block of the cluster (an address of in_block).
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
constexpr uint64_t kWaitNs = 4000000000ull;   // a wait that lasts longer has failed

// Waits for the phase of `parity` to complete; false when it did not within kWaitNs.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    uint64_t began = 0;
    for (uint32_t i = 0;; ++i) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                     "selp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if (i % 64 == 63) {
            const uint64_t t = now_ns();
            if (!began) began = t;
            else if (t - began > kWaitNs) return false;
        }
    }
}

// ------------------------------------------------------------------ whole sectors
// 32 bytes at once: a warp whose lanes write 32 rows writes whole sectors of each.
__device__ __forceinline__ void store32(void *p, const uint32_t (&q)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(q[0]), "r"(q[1]), "r"(q[2]),
                 "r"(q[3]), "r"(q[4]), "r"(q[5]), "r"(q[6]), "r"(q[7]) : "memory");
}
__device__ __forceinline__ void load32(uint32_t (&q)[8], const void *p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]), "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7])
                 : "l"(p) : "memory");
}

// ------------------------------------------------------------------ tensor copies
// Box of `map` at (x, y, z) into this block's shared memory at `dst`; its bytes are counted on
// `bar`, which may be the other block's.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t x, int32_t y,
                                         int32_t z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ------------------------------------------------------------------ tcgen05, two blocks
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"((uint32_t)add) : "memory");
}
// Arrives at `bar` of both blocks once the products issued so far are done.
__device__ __forceinline__ void commit_both(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// 32 or 64 columns of this warp's 32 lanes. One statement loads and waits, so that no use of the
// registers can be moved between the two.
__device__ __forceinline__ void tmem_load(float (&v)[32], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]),
                   "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
                   "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]),
                   "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
                   "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_load(float (&v)[2][32], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
                 "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
                 "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0][0]), "=f"(v[0][1]), "=f"(v[0][2]), "=f"(v[0][3]),
                   "=f"(v[0][4]), "=f"(v[0][5]), "=f"(v[0][6]), "=f"(v[0][7]),
                   "=f"(v[0][8]), "=f"(v[0][9]), "=f"(v[0][10]), "=f"(v[0][11]),
                   "=f"(v[0][12]), "=f"(v[0][13]), "=f"(v[0][14]), "=f"(v[0][15]),
                   "=f"(v[0][16]), "=f"(v[0][17]), "=f"(v[0][18]), "=f"(v[0][19]),
                   "=f"(v[0][20]), "=f"(v[0][21]), "=f"(v[0][22]), "=f"(v[0][23]),
                   "=f"(v[0][24]), "=f"(v[0][25]), "=f"(v[0][26]), "=f"(v[0][27]),
                   "=f"(v[0][28]), "=f"(v[0][29]), "=f"(v[0][30]), "=f"(v[0][31]),
                   "=f"(v[1][0]), "=f"(v[1][1]), "=f"(v[1][2]), "=f"(v[1][3]),
                   "=f"(v[1][4]), "=f"(v[1][5]), "=f"(v[1][6]), "=f"(v[1][7]),
                   "=f"(v[1][8]), "=f"(v[1][9]), "=f"(v[1][10]), "=f"(v[1][11]),
                   "=f"(v[1][12]), "=f"(v[1][13]), "=f"(v[1][14]), "=f"(v[1][15]),
                   "=f"(v[1][16]), "=f"(v[1][17]), "=f"(v[1][18]), "=f"(v[1][19]),
                   "=f"(v[1][20]), "=f"(v[1][21]), "=f"(v[1][22]), "=f"(v[1][23]),
                   "=f"(v[1][24]), "=f"(v[1][25]), "=f"(v[1][26]), "=f"(v[1][27]),
                   "=f"(v[1][28]), "=f"(v[1][29]), "=f"(v[1][30]), "=f"(v[1][31])
                 : "r"(addr) : "memory");
}

// Shared-memory descriptor of a 128-byte-swizzled operand tile of 16-bit elements. Rows that run
// along the summed index: groups of 8 rows lie 1024 bytes apart (the leading offset is unused).
// Rows that run along the other index: groups of 8 rows (of the summed index) lie 1024 bytes
// apart, blocks of 64 elements `block` bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool summed_rows, uint32_t block) {
    const uint64_t lead = summed_rows ? 1 : block >> 4;
    return (uint64_t)((addr >> 4) & 0x3fff) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor: bfloat16 operands, float32 sums, M x N; a_other, b_other where the
// operand's rows run along the index that is not summed.
constexpr uint32_t product_of(int M, int N, bool a_other, bool b_other) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a_other << 15 | (uint32_t)b_other << 16 |
           (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}

}  // namespace tc
}  // namespace dendsn
