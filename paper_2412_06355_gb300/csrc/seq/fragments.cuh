// Products of 16-bit tiles on the warp's matrix instruction, and float32 values as sums of bfloat16
// terms: three terms hold a float32 to 2^-24, two to 2^-17.
//
// A tile lies in shared and in global memory as 8 x 8 blocks of 128 bytes, block rows one after
// another. A block is what eight lanes' 16-byte rows of a matrix load fetch without bank conflicts,
// and what a warp's registers of a product (a pair of neighbours a lane) write as 128 bytes in a row.
// A tile of `t` terms is t such tiles, the leading terms first.
#pragma once

#include <stdint.h>

#include "pieces.cuh"
#include "tc.cuh"

namespace dendsn {

constexpr int kCell = 128;                 // bytes of an 8 x 8 block

// Terms of a pair of values: x = sum of the terms' values, up to what the last one rounds off.
template <int N>
__device__ __forceinline__ void split(uint32_t (&q)[N], float x, float y) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q[i] = bf16_pair(x, y);
        if (i + 1 < N) {
            x -= bf16_low(q[i]);
            y -= bf16_high(q[i]);
        }
    }
}
// What a product of 16 rows and 16 columns of its left factor takes, from two neighbouring results.
template <int N>
__device__ __forceinline__ void split_left(uint32_t (&a)[N][4], const float (&lo)[4], const float (&hi)[4]) {
    uint32_t q[4][N];
    split<N>(q[0], lo[0], lo[1]);
    split<N>(q[1], lo[2], lo[3]);
    split<N>(q[2], hi[0], hi[1]);
    split<N>(q[3], hi[2], hi[3]);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) a[i][j] = q[j][i];
}

__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void fetch4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Right factor, 16 summed places from block `k` and 16 columns from block `n`, of a tile whose rows are
// the columns (`width` blocks a row). r[0], r[1] are the first 8 columns', r[2], r[3] the others'.
__device__ __forceinline__ void right_rows(uint32_t (&r)[4], uint32_t tile, int width, int n, int k) {
    const int lane = threadIdx.x & 31, m = lane >> 3;
    fetch4(r, tile + ((n + (m >> 1)) * width + k + (m & 1)) * kCell + (lane & 7) * 16);
}
// Left factor, 16 rows from block `i` and 16 summed places from block `k`, of a tile whose rows are the rows.
__device__ __forceinline__ void left_rows(uint32_t (&a)[4], uint32_t tile, int width, int i, int k) {
    const int lane = threadIdx.x & 31, m = lane >> 3;
    fetch4(a, tile + ((i + (m & 1)) * width + k + (m >> 1)) * kCell + (lane & 7) * 16);
}

// Adds to the 16 x 16 results c0, c1 the product of a left factor in NA terms and a right one in NB: the
// products of terms i and j with i + j < KEEP, the smallest first, summed by themselves. The matrix
// instruction cuts its sums off where it should round them: a long sum in one accumulator lost up to
// 2e-6 of its norm, this way (one addition of float32 each 16 summed places) 2e-7.
template <int NA, int NB, int KEEP>
__device__ __forceinline__ void products(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[NA][4], const uint32_t (&f)[NB][4]) {
    float t0[4] = {}, t1[4] = {};
#pragma unroll
    for (int sum = KEEP - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = sum - i;
            if (j < 0 || j >= NB) continue;
            multiply(t0, a[i], f[j < 0 || j >= NB ? 0 : j][0], f[j < 0 || j >= NB ? 0 : j][1]);
            multiply(t1, a[i], f[j < 0 || j >= NB ? 0 : j][2], f[j < 0 || j >= NB ? 0 : j][3]);
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) c0[e] += t0[e], c1[e] += t1[e];
}

// `bytes` (a multiple of 16) from global into this block's shared memory, counted on `bar`.
__device__ __forceinline__ void load_bytes(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

}  // namespace dendsn
