// Embedding lookup with scaling (forward) and its gradient by sorted tokens:
// out[i] = scale * table[ids[i]], grad_table[v] = scale * sum of grad_out[i] over ids[i] = v
// in ascending i.
//
// Both are bound by memory: the forward reads and writes n D elements, the backward reads n D
// and writes all V D of the table's gradient. A warp moves one row, four 16-byte vectors of a
// lane in flight. Measured, 131072 tokens of a vocabulary of 131072, D = 2048, bfloat16: forward
// 110 us (5.9 TB/s of DRAM traffic), backward 230 us (the sum 198 us at 5.1 TB/s, the index 27 us);
// 16384 tokens, 50000 rows, D = 1024: 6.4 and 58 us.
//
// The gradient needs each row's positions in a fixed order, so that its float32 sum is the
// same from run to run. They are found by counting: a slot for every token (integer atomics
// in any order), offsets by a prefix sum over the vocabulary, positions scattered to offset +
// slot, and then each row's few positions put in ascending order, by rank within a warp up to
// 32 of them, and by a bitmap of positions in shared memory above. All of that is one launch
// whose blocks meet between the steps: a cluster of 8 up to kFewTokens tokens (its barrier is
// the hardware's), a cooperative grid above. Text has a few tokens with thousands of positions;
// those rows are summed in tiles of 32 positions by one warp each, whose float32 sums are joined
// in order, so that no row waits for one warp. The other rows go 8 to a warp, their positions
// batched across rows so that four gradient rows are in flight whatever the counts are.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "embed_plan.h"
#include "seq_common.h"

namespace dendsn {
namespace {

constexpr int kFew = 32;          // positions a warp orders by rank
constexpr int kTile = 32;         // positions of one partial sum of a longer row
constexpr int kThreads = kIndexThreads;
constexpr int kMapBits = 1 << 20; // positions one pass of the bitmap covers (128 KB)
constexpr int kRowsOfWarp = 8;      // vocabulary rows of a warp of the sum

// VEC elements: 16 bytes where rows and tensors are aligned to 16 bytes, else one element.
template <typename T, int VEC> struct Piece;
template <> struct Piece<float, 4> {
    using Raw = float4;
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    static __device__ __forceinline__ Raw pack(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Piece<float, 1> {
    using Raw = float;
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[1]) { v[0] = r; }
    static __device__ __forceinline__ Raw pack(const float (&v)[1]) { return v[0]; }
};
template <> struct Piece<__nv_bfloat16, 8> {
    using Raw = uint4;
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[8]) {
        const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(q[i] << 16);
            v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ Raw pack(const float (&v)[8]) {
        uint32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            q[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        return make_uint4(q[0], q[1], q[2], q[3]);
    }
};
template <> struct Piece<__nv_bfloat16, 1> {
    using Raw = uint16_t;
    static __device__ __forceinline__ void unpack(const Raw &r, float (&v)[1]) { v[0] = __uint_as_float((uint32_t)r << 16); }
    static __device__ __forceinline__ Raw pack(const float (&v)[1]) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v[0]);
        return *reinterpret_cast<const uint16_t *>(&h);
    }
};

// Work that one warp does on a row at a time: kAhead vectors of each lane.
constexpr int kAhead = 4;

template <typename T, typename I, int VEC>
__global__ void __launch_bounds__(256) embed_forward_kernel(const T *table, const I *ids, T *out, int64_t n,
                                                            int64_t V, int32_t nv, int32_t chunks, int64_t pad,
                                                            float scale) {
    using P = Piece<T, VEC>;
    using Raw = typename P::Raw;
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t i = task / chunks;
    if (i >= n) return;
    const int32_t k0 = (int32_t)(task % chunks) * 32 * kAhead + lane;
    const int64_t id = ids[i];
    Raw *to = reinterpret_cast<Raw *>(out) + i * nv;
    if (id < 0 || id >= V || id == pad) {
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = id == pad && pad >= 0 ? 0.f : __int_as_float(0x7fffffff);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + 32 * j < nv) __stcs(to + k0 + 32 * j, P::pack(v));
        return;
    }
    const Raw *from = reinterpret_cast<const Raw *>(table) + id * nv;
    Raw r[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (k0 + 32 * j < nv) r[j] = __ldg(from + k0 + 32 * j);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
        if (k0 + 32 * j < nv) {
            float v[VEC];
            P::unpack(r[j], v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] *= scale;
            __stcs(to + k0 + 32 * j, P::pack(v));
        }
}

// ------------------------------------------------------------------ positions by row
struct Index {
    int64_t n, V, pad;
    int32_t chunk;       // vocabulary rows whose prefix sums one block forms
    int32_t words;       // of the bitmap
    int32_t *count;      // [V] tokens of a row
    unsigned long long *heads;   // long rows (high half) and their tiles (low half)
    int32_t *base;       // [blocks] tokens of each chunk, then before it
    int32_t *offset;     // [V] tokens before a row within its chunk
    int32_t *slot;       // [n]
    int32_t *pos;        // [n] positions by row
    int32_t *long_row;   // [longs] rows with more than kFew tokens
    int32_t *long_tile;  // [longs] their first tile
    int32_t *tile_of;    // [tiles] the long row (its place in the list) of each tile
    float *partial;      // [tiles][D]
};

__device__ __forceinline__ int32_t first_of(const Index &x, int64_t v) {
    return x.offset[v] + x.base[v / x.chunk];
}
__device__ __forceinline__ int32_t long_rows(const Index &x) { return (int32_t)(*x.heads >> 32); }
__device__ __forceinline__ int32_t long_tiles(const Index &x) { return (int32_t)*x.heads; }

template <typename I> __device__ __forceinline__ int64_t row_of(const I *ids, int64_t i, int64_t V, int64_t pad) {
    const int64_t id = ids[i];
    return id < 0 || id >= V || id == pad ? -1 : id;
}

// Exclusive prefix sum of one value of each of the block's threads, and the sum of all.
__device__ __forceinline__ int32_t prefix(int32_t v, int32_t *warps, int32_t &all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int32_t w = warps[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t u = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += u;
        }
        warps[lane] = w;
    }
    __syncthreads();
    all = warps[31];
    return incl - v + (warp ? warps[warp - 1] : 0);
}

// CLUSTER: the grid is one cluster.
template <typename I, bool CLUSTER>
__global__ void __launch_bounds__(kThreads) embed_index_kernel(const I *ids, Index x) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // embed_sum_kernel comes up
    namespace cg = cooperative_groups;
    auto meet = [] {
        if constexpr (CLUSTER) cg::this_cluster().sync();
        else cg::this_grid().sync();
    };
    extern __shared__ uint32_t map[];
    __shared__ int32_t warps[32];
    const int lane = threadIdx.x & 31;
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, stride = (int64_t)gridDim.x * kThreads;

    for (int64_t v = at; v < x.V; v += stride) x.count[v] = 0;
    if (at == 0) *x.heads = 0;
    meet();

    // A slot of its own for every token among those of its row; one atomic for the equal tokens
    // of a warp. Which token gets which slot depends on the schedule, the set of slots does not.
    for (int64_t i0 = at - lane; i0 < x.n; i0 += stride) {
        const int64_t i = i0 + lane, v = i < x.n ? row_of(ids, i, x.V, x.pad) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, (int)v);
        if (v >= 0) {
            const int leader = __ffs(same) - 1;
            int first = 0;
            if (lane == leader) first = atomicAdd(x.count + v, __popc(same));
            x.slot[i] = __shfl_sync(same, first, leader) + __popc(same & ((1u << lane) - 1));
        }
        __syncwarp();
    }
    meet();

    // Prefix sums of the counts within the block's chunk of rows. Rows with more than kFew tokens
    // are listed with their tiles (the order of the list does not matter to any result).
    {
        const int64_t v0 = (int64_t)blockIdx.x * x.chunk, v1 = min(x.V, v0 + x.chunk);
        int32_t done = 0;
        for (int64_t u = v0; u < v1; u += 4 * kThreads) {
            const int64_t v = u + threadIdx.x * 4;
            int32_t c[4], sum = 0, all;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = v + j < v1 ? __ldcg(x.count + v + j) : 0;
                sum += c[j];
            }
            int32_t before = done + prefix(sum, warps, all);
            done += all;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (v + j < v1) x.offset[v + j] = before;
                before += c[j];
                if (c[j] > kFew) {
                    const unsigned tiles = (unsigned)(c[j] + kTile - 1) / kTile;
                    const unsigned long long h = atomicAdd(x.heads, (1ull << 32) + tiles);
                    x.long_row[h >> 32] = (int32_t)(v + j);
                    x.long_tile[h >> 32] = (int32_t)h;
                }
            }
        }
        if (threadIdx.x == 0) x.base[blockIdx.x] = done;
    }
    meet();

    // The chunks' own prefix sums: every block forms them for itself, block 0 also for later.
    __shared__ int32_t base[kThreads];
    {
        int32_t all;
        const int32_t mine = threadIdx.x < gridDim.x ? __ldcg(x.base + threadIdx.x) : 0;
        base[threadIdx.x] = prefix(mine, warps, all);
        __syncthreads();
    }
    for (int64_t i = at; i < x.n; i += stride) {
        const int64_t v = row_of(ids, i, x.V, x.pad);
        if (v >= 0) x.pos[__ldcg(x.offset + v) + base[v / x.chunk] + x.slot[i]] = (int32_t)i;
    }
    meet();
    if (blockIdx.x == 0 && threadIdx.x < gridDim.x) x.base[threadIdx.x] = base[threadIdx.x];

    // Puts the positions of each long row in ascending order: one bit for each position of the
    // call, set and read back in order. Few tokens: a warp for each row, with a bitmap of its own;
    // else a block, kMapBits positions at a time.
    const int32_t longs = (int32_t)(__ldcg(x.heads) >> 32);
    if constexpr (CLUSTER) {
        const int warp = threadIdx.x >> 5;
        uint32_t *mine = map + warp * x.words;
        for (int k = blockIdx.x * 32 + warp; k < longs; k += gridDim.x * 32) {
            const int32_t v = __ldcg(x.long_row + k), c = __ldcg(x.count + v), tile = __ldcg(x.long_tile + k);
            for (int32_t t = lane; t < (c + kTile - 1) / kTile; t += 32) x.tile_of[tile + t] = k;
            int32_t *pos = x.pos + __ldcg(x.offset + v) + base[v / x.chunk];
            for (int w = lane; w < x.words; w += 32) mine[w] = 0;
            __syncwarp();
            for (int32_t j = lane; j < c; j += 32) {
                const int32_t q = __ldcg(pos + j);
                atomicOr(mine + (q >> 5), 1u << (q & 31));
            }
            __syncwarp();
            const int per = (x.words + 31) / 32, w0 = min(x.words, lane * per), w1 = min(x.words, w0 + per);
            int32_t here = 0;
            for (int w = w0; w < w1; ++w) here += __popc(mine[w]);
            int32_t to = here;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int32_t u = __shfl_up_sync(0xffffffffu, to, o);
                if (lane >= o) to += u;
            }
            to -= here;
            for (int w = w0; w < w1; ++w)
                for (uint32_t m = mine[w]; m; m &= m - 1) pos[to++] = 32 * w + __ffs(m) - 1;
            __syncwarp();
        }
    } else {
        for (int k = blockIdx.x; k < longs; k += gridDim.x) {
            const int32_t v = __ldcg(x.long_row + k), c = __ldcg(x.count + v), tile = __ldcg(x.long_tile + k);
            for (int32_t t = threadIdx.x; t < (c + kTile - 1) / kTile; t += kThreads) x.tile_of[tile + t] = k;
            const int64_t first = __ldcg(x.offset + v) + base[v / x.chunk];
            int32_t *pos = x.pos + first;
            int32_t done = 0;
            // the row's positions are read again for every stretch and overwritten by it only up
            // to the number found so far, so calls of more than one stretch keep them in slot
            const int32_t *src = pos;
            if (x.n > kMapBits) {
                for (int32_t j = threadIdx.x; j < c; j += kThreads) x.slot[first + j] = __ldcg(pos + j);
                src = x.slot + first;
                __syncthreads();
            }
            for (int64_t p0 = 0; p0 < x.n; p0 += kMapBits) {
                for (int w = threadIdx.x; w < x.words; w += kThreads) map[w] = 0;
                __syncthreads();
                for (int32_t j = threadIdx.x; j < c; j += kThreads) {
                    const int64_t p = __ldcg(src + j) - p0;
                    if (p >= 0 && p < kMapBits) atomicOr(map + (p >> 5), 1u << (p & 31));
                }
                __syncthreads();
                // each thread reads back `per` consecutive words
                const int per = (x.words + kThreads - 1) / kThreads, w0 = threadIdx.x * per, w1 = min(x.words, w0 + per);
                int32_t mine = 0, all;
                for (int w = w0; w < w1; ++w) mine += __popc(map[w]);
                int32_t to = done + prefix(mine, warps, all);
                done += all;
                for (int w = w0; w < w1; ++w)
                    for (uint32_t m = map[w]; m; m &= m - 1) pos[to++] = (int32_t)(p0 + 32 * w + __ffs(m) - 1);
                __syncthreads();
            }
        }
    }
}

// Adds up gradient rows, `m` of them at the positions `p` of the warp's lanes in order, four in
// flight, for the kAhead vectors from k0 on; calls done(k, sums) after each position k whose bit
// is set in `ends`, and begins anew.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void add_rows(const T *grad, int32_t nv, int32_t k0, int32_t p, int m, uint32_t ends, F done) {
    using P = Piece<T, VEC>;
    using Raw = typename P::Raw;
    constexpr int kRows = 4;
    float acc[kAhead][VEC] = {};
    for (int k = 0; k < m; k += kRows) {
        Raw r[kRows][kAhead];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const Raw *from = reinterpret_cast<const Raw *>(grad) + (int64_t)__shfl_sync(0xffffffffu, p, min(k + u, 31)) * nv;
            if (k + u < m)
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (k0 + 32 * j < nv) r[u][j] = __ldcs(from + k0 + 32 * j);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            if (k + u < m) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (k0 + 32 * j < nv) {
                        float v[VEC];
                        P::unpack(r[u][j], v);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) acc[j][e] += v[e];
                    }
                if (ends >> (k + u) & 1) {
                    done(k + u, acc);
#pragma unroll
                    for (int j = 0; j < kAhead; ++j)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) acc[j][e] = 0.f;
                }
            }
    }
}

// One warp per task: first the tiles of long rows, then kRowsOfWarp rows of the vocabulary each.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) embed_sum_kernel(const T *grad, T *gtable, Index x, int64_t D, int32_t nv,
                                                        float scale) {
    using P = Piece<T, VEC>;
    using Raw = typename P::Raw;
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int32_t tiles = x.n > kFew ? long_tiles(x) : 0;
    if (task < tiles) {
        const int32_t at = x.tile_of[task], v = x.long_row[at], k = (int32_t)task - x.long_tile[at];
        const int32_t c = min(kTile, x.count[v] - k * kTile);
        const int32_t p = lane < c ? x.pos[first_of(x, v) + k * kTile + lane] : 0;
        float *part = x.partial + task * D;
        for (int32_t k0 = lane; k0 - lane < nv; k0 += 32 * kAhead)
            add_rows<T, VEC>(grad, nv, k0, p, c, 1u << (c - 1), [&](int, float (&acc)[kAhead][VEC]) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (k0 + 32 * j < nv)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) part[(int64_t)(k0 + 32 * j) * VEC + e] = acc[j][e];
            });
        return;
    }
    const int64_t v0 = (task - tiles) * kRowsOfWarp;
    if (v0 >= x.V) return;
    const bool row = lane < kRowsOfWarp && v0 + lane < x.V;
    const int32_t all = row && x.n > 0 ? x.count[v0 + lane] : 0, c = all > kFew ? 0 : all;
    const int32_t first = c ? first_of(x, v0 + lane) : 0;
    // rows without tokens
    for (uint32_t m = __ballot_sync(0xffffffffu, row && all == 0); m; m &= m - 1) {
        Raw *to = reinterpret_cast<Raw *>(gtable) + (v0 + __ffs(m) - 1) * nv;
        float zero[VEC] = {};
        for (int32_t k = lane; k < nv; k += 32) __stcs(to + k, P::pack(zero));
    }
    int32_t incl = c;
#pragma unroll
    for (int o = 1; o < kRowsOfWarp; o <<= 1) {
        const int32_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    // batches of rows with up to 32 positions together
    const int32_t total = __shfl_sync(0xffffffffu, incl, kRowsOfWarp - 1);
    for (int32_t done = 0; done < total;) {
        const uint32_t fits = __ballot_sync(0xffffffffu, lane < kRowsOfWarp && incl - done <= 32);
        const int last = 31 - __clz(fits);                   // the batch's last row
        const int m = __shfl_sync(0xffffffffu, incl, last) - done;
        // lane i takes the batch's position i: its row is the first whose end lies beyond i
        int mine = 0;
#pragma unroll
        for (int r = 0; r < kRowsOfWarp; ++r) mine += __shfl_sync(0xffffffffu, incl, r) - done <= lane;
        mine = min(mine, kRowsOfWarp - 1);
        const int32_t end = __shfl_sync(0xffffffffu, incl, mine) - done, size = __shfl_sync(0xffffffffu, c, mine);
        const int32_t from = __shfl_sync(0xffffffffu, first, mine), start = end - size;
        const int32_t q = lane < m ? x.pos[from + lane - start] : 0;
        // its place among its row's positions in ascending order
        int rank = start;
        for (int k = 0; k < m; ++k) {
            const int32_t other = __shfl_sync(0xffffffffu, q, k);
            rank += k >= start && k < end && other < q;
        }
        int32_t p = 0;
        for (int k = 0; k < m; ++k) {
            const int32_t other = __shfl_sync(0xffffffffu, q, k), r = __shfl_sync(0xffffffffu, rank, k);
            if (r == lane) p = other;
        }
        const uint32_t ends = __ballot_sync(0xffffffffu, lane < m && lane == end - 1);
        for (int32_t k0 = lane; k0 - lane < nv; k0 += 32 * kAhead)
            add_rows<T, VEC>(grad, nv, k0, p, m, ends, [&](int k, float (&acc)[kAhead][VEC]) {
                Raw *to = reinterpret_cast<Raw *>(gtable) + (v0 + __shfl_sync(0xffffffffu, mine, k)) * nv;
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (k0 + 32 * j < nv) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) acc[j][e] *= scale;
                        __stcs(to + k0 + 32 * j, P::pack(acc[j]));
                    }
            });
        done += m;
    }
}

// Joins the tiles of the long rows in order: blocks of 256 columns of one row.
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(T *gtable, Index x, int64_t D, float scale) {
    pdl_begin();
    const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (d >= D) return;
    const int32_t longs = long_rows(x);
    for (int at = blockIdx.y; at < longs; at += gridDim.y) {
        const int32_t v = x.long_row[at], tiles = (x.count[v] + kTile - 1) / kTile;
        const float *p = x.partial + (int64_t)x.long_tile[at] * D + d;
        float sum = 0.f;
        int k = 0;
        for (; k + 8 <= tiles; k += 8) {
            float r[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) r[u] = p[(int64_t)(k + u) * D];
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += r[u];
        }
        for (; k < tiles; ++k) sum += p[(int64_t)k * D];
        float o[1] = {sum * scale};
        reinterpret_cast<typename Piece<T, 1>::Raw *>(gtable)[v * D + d] = Piece<T, 1>::pack(o);
    }
}

// SMs of the current device.
int device_sms() {
    int dev = 0, n = 0;
    const bool ok = cudaGetDevice(&dev) == cudaSuccess &&
                    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0;
    return ok ? n : 1;
}

struct Plan {
    int64_t longs, tiles;         // most long rows and tiles there can be
    size_t at[10], scratch;
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
    if (!std::isfinite(cfg->scale)) return seq_fail(DENDSN_ERR_INVALID_ARG, "scale must be finite");
    // the largest grids: a warp for every kAhead vectors of an output row, and for every row and tile
    if ((cfg->n * (((int64_t)cfg->D + 32 * kAhead - 1) / (32 * kAhead)) + 7) / 8 > INT32_MAX)
        return seq_fail(DENDSN_ERR_UNSUPPORTED, "too many elements (n=%lld D=%d)", (long long)cfg->n, cfg->D);
    pl->longs = std::min<int64_t>(cfg->V, cfg->n / (kFew + 1));
    pl->tiles = cfg->n / kTile + pl->longs;
    const size_t sizes[10] = {(size_t)cfg->V * 4, 16, kMostIndexBlocks * 4, (size_t)cfg->V * 4, (size_t)cfg->n * 4,
                              (size_t)cfg->n * 4, (size_t)pl->longs * 4, (size_t)pl->longs * 4, (size_t)pl->tiles * 4,
                              (size_t)pl->tiles * cfg->D * 4};
    size_t at = 0;
    for (int i = 0; i < 10; ++i) {
        pl->at[i] = at;
        at += (sizes[i] + 15) / 16 * 16;
    }
    pl->scratch = at;
    return DENDSN_OK;
}

template <typename T, typename I, int VEC>
cudaError_t run_forward(const dendsn_embed_config &c, const void *table, const void *ids, void *out,
                        cudaStream_t s) {
    const int32_t nv = c.D / VEC, chunks = (nv + 32 * kAhead - 1) / (32 * kAhead);
    const int64_t blocks = (c.n * chunks + 7) / 8;
    return seq_launch(embed_forward_kernel<T, I, VEC>, dim3((unsigned)blocks), 256, 0, s, 1, static_cast<const T *>(table),
                      static_cast<const I *>(ids), static_cast<T *>(out), c.n, c.V, nv, chunks, c.padding_id, c.scale);
}

template <typename T, typename I, int VEC>
cudaError_t run_backward(const dendsn_embed_config &c, const Plan &pl, const void *ids_, const void *grad,
                         void *gtable, void *scratch, cudaStream_t s, int *launches) {
    char *p = static_cast<char *>(scratch);
    auto ints = [&](int i) { return reinterpret_cast<int32_t *>(p + pl.at[i]); };
    const IndexGrid grid = index_grid(c.n, c.V, device_sms());
    Index x{c.n, c.V, c.padding_id, grid.chunk, (int32_t)(std::min<int64_t>(c.n, kMapBits) + 31) / 32, ints(0),
            reinterpret_cast<unsigned long long *>(p + pl.at[1]), ints(2), ints(3), ints(4), ints(5), ints(6), ints(7),
            ints(8), reinterpret_cast<float *>(p + pl.at[9])};
    const I *ids = static_cast<const I *>(ids_);
    const T *g = static_cast<const T *>(grad);
    T *gt = static_cast<T *>(gtable);
    const int32_t nv = c.D / VEC;
    if (c.n > 0) {
        const bool few = grid.cluster;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)grid.blocks);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = pl.longs > 0 ? (size_t)x.words * 4 * (few ? kThreads / 32 : 1) : 0;
        cfg.stream = s;
        cudaLaunchAttribute at[1];
        if (few) {
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = (unsigned)grid.blocks;
            at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        } else {
            at[0].id = cudaLaunchAttributeCooperative;
            at[0].val.cooperative = 1;
        }
        cfg.attrs = at;
        cfg.numAttrs = 1;
        auto start = [&](auto kernel) {
            // the limit is the kernel's, not the call's: always the largest, so that no other host
            // thread lowers it before this launch
            if (cfg.dynamicSmemBytes > 32768) {
                cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMapBits / 8);
                if (e != cudaSuccess) return e;
            }
            return cudaLaunchKernelEx(&cfg, kernel, ids, x);
        };
        cudaError_t e = few ? start(embed_index_kernel<I, true>) : start(embed_index_kernel<I, false>);
        if (e != cudaSuccess) return e;
        *launches += 1;
    }
    const int64_t warps = (c.V + kRowsOfWarp - 1) / kRowsOfWarp + pl.tiles;
    cudaError_t e = seq_launch(embed_sum_kernel<T, VEC>, dim3((unsigned)((warps + 7) / 8)), 256, 0, s, 1, g, gt, x, c.D, nv, c.scale);
    *launches += 1;
    if (e == cudaSuccess && pl.longs > 0) {
        const dim3 columns((unsigned)((c.D + 255) / 256), (unsigned)std::min<int64_t>(pl.longs, 1024));
        e = seq_launch(embed_join_kernel<T>, columns, 256, 0, s, 1, gt, x, c.D, c.scale);
        *launches += 1;
    }
    return e;
}

// Whether rows of D elements of every tensor can be taken 16 bytes at a time.
bool wide(const dendsn_embed_config &c, const void *a, const void *b) {
    const size_t sx = c.x_dtype == DENDSN_BF16 ? 2 : 4;
    return c.D * sx % 16 == 0 && seq_aligned(a, 16) && seq_aligned(b, 16);
}

template <typename T, typename I>
cudaError_t pick_forward(const dendsn_embed_config &c, const void *table, const void *ids, void *out, cudaStream_t s) {
    return wide(c, table, out) ? run_forward<T, I, 16 / sizeof(T)>(c, table, ids, out, s)
                               : run_forward<T, I, 1>(c, table, ids, out, s);
}
template <typename T, typename I>
cudaError_t pick_backward(const dendsn_embed_config &c, const Plan &pl, const void *ids, const void *grad,
                          void *gtable, void *scratch, cudaStream_t s, int *launches) {
    return wide(c, grad, gtable) ? run_backward<T, I, 16 / sizeof(T)>(c, pl, ids, grad, gtable, scratch, s, launches)
                                 : run_backward<T, I, 1>(c, pl, ids, grad, gtable, scratch, s, launches);
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
    cudaError_t e = bf ? (i64 ? pick_forward<__nv_bfloat16, int64_t>(*cfg, table, ids, out, s)
                              : pick_forward<__nv_bfloat16, int32_t>(*cfg, table, ids, out, s))
                       : (i64 ? pick_forward<float, int64_t>(*cfg, table, ids, out, s)
                              : pick_forward<float, int32_t>(*cfg, table, ids, out, s));
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
    if (!scratch) return seq_fail(DENDSN_ERR_INVALID_ARG, "scratch is NULL");
    if (!seq_aligned(scratch, 16)) return seq_fail(DENDSN_ERR_MISALIGNED, "scratch must be 16-byte aligned");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int launches = 0;
    cudaError_t e = bf ? (i64 ? pick_backward<__nv_bfloat16, int64_t>(*cfg, pl, ids, grad_out, grad_table, scratch, s, &launches)
                              : pick_backward<__nv_bfloat16, int32_t>(*cfg, pl, ids, grad_out, grad_table, scratch, s, &launches))
                       : (i64 ? pick_backward<float, int64_t>(*cfg, pl, ids, grad_out, grad_table, scratch, s, &launches)
                              : pick_backward<float, int32_t>(*cfg, pl, ids, grad_out, grad_table, scratch, s, &launches));
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "embed backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(launches);
    return DENDSN_OK;
}

}  // extern "C"
