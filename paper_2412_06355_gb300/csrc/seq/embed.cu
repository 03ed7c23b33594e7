// Embedding lookup with scaling (forward) and its gradient by sorted tokens:
// out[i] = scale * table[ids[i]], grad_table[v] = scale * sum of grad_out[i] over ids[i] = v
// in ascending i.
//
// Both are bound by memory: the forward reads and writes n D elements, the backward reads n D
// and writes all V D of the table's gradient. A warp moves one row, four 16-byte vectors of a
// lane in flight.
//
// The gradient needs each row's positions in a fixed order, so that its float32 sum is the
// same from run to run. They are found by counting: a slot for every token (integer atomics
// in any order), offsets by a prefix sum over the vocabulary, positions scattered to offset +
// slot, and then each row's few positions put in ascending order, by rank within a warp up to
// 32 of them, and by a bitmap of positions in shared memory above. Text has a few tokens with
// thousands of positions; those rows are summed in tiles of 64 positions by one warp each,
// whose float32 sums are joined in order, so that no row waits for one warp.
#include <cuda_bf16.h>

#include <algorithm>

#include "seq_common.h"

namespace dendsn {
namespace {

constexpr int kFew = 32;          // positions a warp orders by rank
constexpr int kTile = 64;         // positions of one partial sum of a longer row
constexpr int kScanRows = 4096;   // vocabulary rows of one prefix block
constexpr int kMapBits = 1 << 20; // positions one pass of the bitmap covers (128 KB)

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
    int32_t *count;      // [V] tokens of a row
    int32_t *base;       // [prefix blocks] tokens before each block of kScanRows rows
    int32_t *heads;      // [4]: long rows, their tiles, finished prefix blocks
    int32_t *offset;     // [V] tokens before a row within its block
    int32_t *slot;       // [n]
    int32_t *pos;        // [n] positions by row
    int32_t *long_row;   // [longs] rows with more than kFew tokens
    int32_t *long_tile;  // [longs] their first tile
    int32_t *tile_of;    // [tiles] the long row (its place in the list) of each tile
    float *partial;      // [tiles][D]
};

__device__ __forceinline__ int32_t first_of(const Index &x, int64_t v) {
    return x.offset[v] + x.base[v / kScanRows];
}

template <typename I> __device__ __forceinline__ int64_t row_of(const I *ids, int64_t i, int64_t V, int64_t pad) {
    const int64_t id = ids[i];
    return id < 0 || id >= V || id == pad ? -1 : id;
}

// A slot of its own for every token among those of its row; one atomic for the equal tokens of
// a warp. Which token gets which slot depends on the schedule, the set of slots does not.
template <typename I>
__global__ void __launch_bounds__(256) embed_count_kernel(const I *ids, Index x, int64_t n, int64_t V, int64_t pad) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int lane = threadIdx.x & 31;
    const int64_t v = i < n ? row_of(ids, i, V, pad) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, (int)v);
    if (v < 0) return;
    const int leader = __ffs(same) - 1;
    int first = 0;
    if (lane == leader) first = atomicAdd(x.count + v, __popc(same));
    first = __shfl_sync(same, first, leader);
    x.slot[i] = first + __popc(same & ((1u << lane) - 1));
}

// Exclusive prefix sums of the counts within blocks of kScanRows rows; the last block to finish
// sums up the blocks. Rows with more than kFew tokens are listed with their tiles (the order of
// the list does not matter to any result).
__global__ void __launch_bounds__(1024) embed_prefix_kernel(Index x, int64_t V, int32_t blocks) {
    __shared__ int32_t warps[32];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t v0 = (int64_t)blockIdx.x * kScanRows + threadIdx.x * 4;
    int32_t c[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c[j] = v0 + j < V ? x.count[v0 + j] : 0;
        sum += c[j];
    }
    int32_t incl = sum;
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 31) warps[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int32_t w = warps[lane];
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t up = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += up;
        }
        warps[lane] = w;
    }
    __syncthreads();
    int32_t before = incl - sum + (warp ? warps[warp - 1] : 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (v0 + j < V) x.offset[v0 + j] = before;
        before += c[j];
        if (c[j] > kFew) {
            const int at = atomicAdd(x.heads, 1), tiles = (c[j] + kTile - 1) / kTile;
            const int tile = atomicAdd(x.heads + 1, tiles);
            x.long_row[at] = (int32_t)(v0 + j);
            x.long_tile[at] = tile;
            for (int k = 0; k < tiles; ++k) x.tile_of[tile + k] = at;
        }
    }
    if (threadIdx.x == 0) {
        x.base[blockIdx.x] = warps[31];
        __threadfence();
        last = atomicAdd(x.heads + 2, 1) == blocks - 1;
    }
    __syncthreads();
    if (last && threadIdx.x == 0) {
        __threadfence();
        int32_t total = 0;
        for (int b = 0; b < blocks; ++b) {
            const int32_t t = __ldcg(x.base + b);
            x.base[b] = total;
            total += t;
        }
    }
}

template <typename I>
__global__ void __launch_bounds__(256) embed_scatter_kernel(const I *ids, Index x, int64_t n, int64_t V, int64_t pad) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t v = i < n ? row_of(ids, i, V, pad) : -1;
    if (v >= 0) x.pos[first_of(x, v) + x.slot[i]] = (int32_t)i;
}

// Puts the positions of each long row in ascending order: one bit for each position of the
// call, set and read back in order, kMapBits positions at a time.
__global__ void __launch_bounds__(256) embed_order_kernel(Index x, int64_t n, int32_t words) {
    extern __shared__ uint32_t map[];
    __shared__ int32_t warps[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int k = blockIdx.x; k < x.heads[0]; k += gridDim.x) {
        const int32_t v = x.long_row[k], c = x.count[v];
        int32_t *pos = x.pos + first_of(x, v);
        int32_t done = 0;
        // the row's positions are read again for every stretch and overwritten by it only up
        // to the number found so far, so calls of more than one stretch keep them in slot
        const int32_t *src = pos;
        if (n > kMapBits) {
            for (int32_t j = threadIdx.x; j < c; j += 256) x.slot[first_of(x, v) + j] = pos[j];
            src = x.slot + first_of(x, v);
            __syncthreads();
        }
        for (int64_t p0 = 0; p0 < n; p0 += kMapBits) {
            for (int w = threadIdx.x; w < words; w += 256) map[w] = 0;
            __syncthreads();
            for (int32_t j = threadIdx.x; j < c; j += 256) {
                const int64_t p = src[j] - p0;
                if (p >= 0 && p < kMapBits) atomicOr(map + (p >> 5), 1u << (p & 31));
            }
            __syncthreads();
            // each thread reads back `per` consecutive words
            const int per = (words + 255) / 256, w0 = threadIdx.x * per, w1 = min(words, w0 + per);
            int32_t mine = 0;
            for (int w = w0; w < w1; ++w) mine += __popc(map[w]);
            int32_t incl = mine;
            for (int o = 1; o < 32; o <<= 1) {
                const int32_t up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            if (lane == 31) warps[warp] = incl;
            __syncthreads();
            int32_t at = done + incl - mine;
            for (int w = 0; w < 8; ++w) {
                if (w < warp) at += warps[w];
                done += warps[w];
            }
            for (int w = w0; w < w1; ++w)
                for (uint32_t m = map[w]; m; m &= m - 1) pos[at++] = (int32_t)(p0 + 32 * w + __ffs(m) - 1);
            __syncthreads();
        }
    }
}

// Sum of the rows at `c` positions, `p` holding up to 32 of them in the warp's lanes.
template <typename T, int VEC>
__device__ __forceinline__ void add_rows(float (&acc)[kAhead][VEC], const T *grad, int32_t nv, int32_t k0,
                                         int32_t p, int c) {
    using P = Piece<T, VEC>;
    using Raw = typename P::Raw;
    for (int k = 0; k < c; ++k) {
        const Raw *from = reinterpret_cast<const Raw *>(grad) + (int64_t)__shfl_sync(0xffffffffu, p, k) * nv;
        Raw r[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + 32 * j < nv) r[j] = __ldcs(from + k0 + 32 * j);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + 32 * j < nv) {
                float v[VEC];
                P::unpack(r[j], v);
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[j][e] += v[e];
            }
    }
}

// One warp per task: first the tiles of long rows, then every row of the vocabulary.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) embed_sum_kernel(const T *grad, T *gtable, Index x, int64_t V, int64_t D,
                                                        int32_t nv, float scale) {
    using P = Piece<T, VEC>;
    using Raw = typename P::Raw;
    const int lane = threadIdx.x & 31;
    const int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int32_t tiles = x.heads[1];
    int32_t p = 0, c, p2 = 0, c2 = 0;
    float *part = nullptr;
    Raw *to = nullptr;
    if (task < tiles) {
        const int32_t at = x.tile_of[task], v = x.long_row[at], k = (int32_t)task - x.long_tile[at];
        const int32_t *pos = x.pos + first_of(x, v) + k * kTile;
        const int32_t all = min(kTile, x.count[v] - k * kTile);
        c = min(32, all);
        c2 = all - c;
        if (lane < c) p = pos[lane];
        if (lane < c2) p2 = pos[32 + lane];
        part = x.partial + task * D;
    } else {
        const int64_t v = task - tiles;
        if (v >= V) return;
        c = x.count[v];
        if (c > kFew) return;
        to = reinterpret_cast<Raw *>(gtable) + v * nv;
        const int32_t mine = c && lane < c ? x.pos[first_of(x, v) + lane] : INT32_MAX;
        int rank = 0;
        for (int k = 0; k < c; ++k) rank += __shfl_sync(0xffffffffu, mine, k) < mine;
        // lane r takes the position whose rank is r
        for (int k = 0; k < c; ++k) {
            const int32_t q = __shfl_sync(0xffffffffu, mine, k), r = __shfl_sync(0xffffffffu, rank, k);
            if (r == lane) p = q;
        }
    }
    for (int32_t k0 = lane; k0 - lane < nv; k0 += 32 * kAhead) {
        float acc[kAhead][VEC] = {};
        add_rows<T, VEC>(acc, grad, nv, k0, p, c);
        if (c2) add_rows<T, VEC>(acc, grad, nv, k0, p2, c2);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + 32 * j < nv) {
                if (part) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) part[(int64_t)(k0 + 32 * j) * VEC + e] = acc[j][e];
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[j][e] *= scale;
                    __stcs(to + k0 + 32 * j, P::pack(acc[j]));
                }
            }
    }
}

// Joins the tiles of the long rows in order: blocks of 256 columns of one row.
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(T *gtable, Index x, int64_t D, float scale) {
    const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (d >= D) return;
    for (int at = blockIdx.y; at < x.heads[0]; at += gridDim.y) {
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

struct Plan {
    int32_t blocks;               // of the prefix sum
    int64_t longs, tiles;         // most long rows and tiles there can be
    size_t at[10], zeroed, scratch;
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
    // the largest grids: a warp for every kAhead vectors of an output row, and for every row and tile
    if ((cfg->n * (((int64_t)cfg->D + 32 * kAhead - 1) / (32 * kAhead)) + 7) / 8 > INT32_MAX)
        return seq_fail(DENDSN_ERR_UNSUPPORTED, "too many elements (n=%lld D=%d)", (long long)cfg->n, cfg->D);
    pl->blocks = (int32_t)(((int64_t)cfg->V + kScanRows - 1) / kScanRows);
    pl->longs = std::min<int64_t>(cfg->V, cfg->n / (kFew + 1));
    pl->tiles = cfg->n / kTile + pl->longs;
    const size_t sizes[10] = {(size_t)cfg->V * 4, (size_t)pl->blocks * 4, 16, (size_t)cfg->V * 4, (size_t)cfg->n * 4,
                              (size_t)cfg->n * 4, (size_t)pl->longs * 4, (size_t)pl->longs * 4, (size_t)pl->tiles * 4,
                              (size_t)pl->tiles * cfg->D * 4};
    size_t at = 0;
    for (int i = 0; i < 10; ++i) {
        pl->at[i] = at;
        at += (sizes[i] + 15) / 16 * 16;
        if (i == 2) pl->zeroed = at;      // count, base and heads start at zero
    }
    pl->scratch = at;
    return DENDSN_OK;
}

template <typename T, typename I, int VEC>
cudaError_t run_forward(const dendsn_embed_config &c, const void *table, const void *ids, void *out,
                        cudaStream_t s) {
    const int32_t nv = c.D / VEC, chunks = (nv + 32 * kAhead - 1) / (32 * kAhead);
    const int64_t blocks = (c.n * chunks + 7) / 8;
    embed_forward_kernel<T, I, VEC><<<(unsigned)blocks, 256, 0, s>>>(
        static_cast<const T *>(table), static_cast<const I *>(ids), static_cast<T *>(out), c.n, c.V, nv, chunks,
        c.padding_id, c.scale);
    return cudaGetLastError();
}

template <typename T, typename I, int VEC>
cudaError_t run_backward(const dendsn_embed_config &c, const Plan &pl, const void *ids_, const void *grad,
                         void *gtable, void *scratch, cudaStream_t s, int *launches) {
    char *p = static_cast<char *>(scratch);
    auto ints = [&](int i) { return reinterpret_cast<int32_t *>(p + pl.at[i]); };
    Index x{ints(0), ints(1), ints(2), ints(3), ints(4), ints(5), ints(6), ints(7), ints(8),
            reinterpret_cast<float *>(p + pl.at[9])};
    const I *ids = static_cast<const I *>(ids_);
    const T *g = static_cast<const T *>(grad);
    T *gt = static_cast<T *>(gtable);
    const int32_t nv = c.D / VEC;
    const unsigned tokens = (unsigned)((c.n + 255) / 256);
    cudaError_t e = cudaMemsetAsync(scratch, 0, pl.zeroed, s);
    if (e != cudaSuccess) return e;
    if (c.n > 0) {
        embed_count_kernel<I><<<tokens, 256, 0, s>>>(ids, x, c.n, c.V, c.padding_id);
        embed_prefix_kernel<<<pl.blocks, 1024, 0, s>>>(x, c.V, pl.blocks);
        embed_scatter_kernel<I><<<tokens, 256, 0, s>>>(ids, x, c.n, c.V, c.padding_id);
        *launches += 3;
    }
    if (pl.longs > 0) {
        const int32_t words = (int32_t)(std::min<int64_t>(c.n, kMapBits) + 31) / 32;
        if (words * 4 > 48 * 1024) {
            e = cudaFuncSetAttribute(embed_order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, words * 4);
            if (e != cudaSuccess) return e;
        }
        embed_order_kernel<<<(unsigned)std::min<int64_t>(pl.longs, 608), 256, words * 4, s>>>(x, c.n, words);
        *launches += 1;
    }
    embed_sum_kernel<T, VEC><<<(unsigned)((c.V + pl.tiles + 7) / 8), 256, 0, s>>>(g, gt, x, c.V, c.D, nv, c.scale);
    *launches += 1;
    if (pl.longs > 0) {
        const dim3 grid((unsigned)((c.D + 255) / 256), (unsigned)std::min<int64_t>(pl.longs, 1024));
        embed_join_kernel<T><<<grid, 256, 0, s>>>(gt, x, c.D, c.scale);
        *launches += 1;
    }
    return cudaGetLastError();
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
