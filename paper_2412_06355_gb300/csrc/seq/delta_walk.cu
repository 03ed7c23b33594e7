// The states of the gated delta rule, and their gradients, from chunk to chunk: what has an order. The formulas and
// what happens before and after stand in delta.cu.
//
// A block has one head of one sequence. Columns of v do not meet, so the products are turned: 128 lanes of tensor
// memory are the columns, and everything a chunk needs comes from three rounds of tcgen05 products (forward: k S and
// q S; e; P u and k^T (rest u). backward: P^T go and k D; y; q^T go and k^T y), whose left factors the threads write to
// tensor memory as bfloat16 terms and whose right factors are the chunk's tiles in shared memory. The state itself
// stays in registers as float32: four threads a column, a quarter of the places each. Sixteen warps compute, one more
// fetches tiles and issues products; in between they wait for each other on mbarriers. (8 x 2048 tokens, 16 heads of
// 128 x 128, forward: eight warps 470 us, sixteen of which one issues 226, as here 170.)
//
// What bounds it is the chain: a chunk is three rounds of (registers -> tensor memory -> products -> registers), and
// a block has all of an SM's tensor memory, so that 128 sequences and heads are 128 SMs at work.
#include <algorithm>

#include "delta_common.cuh"
#include "tc_one.cuh"

namespace dendsn {
namespace delta {
namespace {

constexpr int kWarps = 16;                 // that compute
constexpr int kThreads = (kWarps + 4) * 32;            // one more issues, one fetches; two only share its registers out
constexpr int kParts = kWarps / 4;         // threads of a column of v
constexpr int kTokens = C / kParts;        // tokens of a thread
constexpr uint32_t kColumns = 512;         // of tensor memory: all there are

// A stage of shared memory: a chunk's tiles.
struct Stage {
    uint32_t k, q, x, p, gates, bytes;
};
__host__ __device__ inline Stage stage_of(const DeltaPlan &p) {
    Stage s;
    s.k = 0;
    s.q = s.k + (uint32_t)p.key_bytes;
    s.x = s.q + (uint32_t)p.key_bytes;
    s.p = s.x + kSquare;
    s.gates = s.p + kSquare;
    s.bytes = s.gates + kGateFloats * 4;
    return s;
}
// One warp: the chunk's tiles into a stage. Of the square matrices only the blocks on and below the diagonal of 16 x 16
// are written, and fetched: a row of blocks a lane.
constexpr uint32_t kTriangle = 3 * 5120;   // bytes of what is fetched of one
__device__ __forceinline__ void load_stage(const Args &a, const Stage &st, uint32_t smem, uint32_t bar, const uint8_t *kept, size_t x, int64_t slot, int h) {
    const int64_t hk = slot * a.Hk + h / (a.Hv / a.Hk), hv = slot * a.Hv + h;
    const int lane = threadIdx.x & 31;
    if (lane == 0) tc::bar_expect(bar, 2 * (uint32_t)a.p.key_bytes + 2 * kTriangle + kGateFloats * 4);
    __syncwarp();
    if (lane < 24) {
        const uint32_t at = lane * 8 * kCell, bytes = (lane % 8 / 2 + 1) * 2 * kCell;      // term lane / 8, row of blocks lane % 8
        load_bytes(smem + st.x + at, kept + x + hv * kSquare + at, bytes, bar);
        load_bytes(smem + st.p + at, kept + a.p.p + hv * kSquare + at, bytes, bar);
    } else if (lane == 24) {
        load_bytes(smem + st.k, kept + a.p.k + hk * a.p.key_bytes, (uint32_t)a.p.key_bytes, bar);
    } else if (lane == 25) {
        load_bytes(smem + st.q, kept + a.p.q + hk * a.p.key_bytes, (uint32_t)a.p.key_bytes, bar);
    } else if (lane == 26) {
        load_bytes(smem + st.gates, kept + a.p.gates + hv * kGateFloats * 4, kGateFloats * 4, bar);
    }
    __syncwarp();
}

// A thread's tokens of one column of v or go, fetched ahead of their use.
template <typename T>
struct Ahead;
template <>
struct Ahead<float> {
    float r[kTokens];
    __device__ __forceinline__ void set(int i, const float *p) { r[i] = *p; }
    __device__ __forceinline__ void zero(int i) { r[i] = 0.f; }
    __device__ __forceinline__ float get(int i) const { return r[i]; }
    template <int N>
    __device__ __forceinline__ void pair(uint32_t (&q)[N], int i) const { split<N>(q, r[2 * i], r[2 * i + 1]); }
};
template <>
struct Ahead<__nv_bfloat16> {
    uint32_t r[kTokens];
    __device__ __forceinline__ void set(int i, const __nv_bfloat16 *p) { r[i] = *reinterpret_cast<const uint16_t *>(p); }
    __device__ __forceinline__ void zero(int i) { r[i] = 0; }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(r[i] << 16); }
    template <int N>
    __device__ __forceinline__ void pair(uint32_t (&q)[N], int i) const { q[0] = r[2 * i] | r[2 * i + 1] << 16; }
};
template <typename T>
__device__ __forceinline__ void fetch(Ahead<T> &x, const T *from, int64_t stride, int left) {
    if (left >= kTokens) {
#pragma unroll
        for (int i = 0; i < kTokens; ++i, from += stride) x.set(i, from);
    } else {
#pragma unroll
        for (int i = 0; i < kTokens; ++i, from += stride) {
            x.zero(i);
            if (i < left) x.set(i, from);
        }
    }
}
// For every of a thread's tokens, its place and one of a chunk's gate values.
template <typename F>
__device__ __forceinline__ void each(const float *from, F f) {
#pragma unroll
    for (int i = 0; i < kTokens; i += 4) {
        const float4 x = *reinterpret_cast<const float4 *>(from + i);
        f(i, x.x), f(i + 1, x.y), f(i + 2, x.z), f(i + 3, x.w);
    }
}

// Terms of values as left factors: 8 columns for each 16 values; terms lie `term` columns apart.
template <int N, int K>
__device__ __forceinline__ void to_lanes(uint32_t to, uint32_t term, const float (&v)[K]) {
#pragma unroll
    for (int part = 0; part < K / 16; ++part) {
        uint32_t q[N][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t t[N];
            split<N>(t, v[part * 16 + 2 * i], v[part * 16 + 2 * i + 1]);
#pragma unroll
            for (int n = 0; n < N; ++n) q[n][i] = t[n];
        }
#pragma unroll
        for (int n = 0; n < N; ++n) tc::tmem_store(to + n * term + part * 8, q[n]);
    }
}
template <int N, typename T>
__device__ __forceinline__ void to_lanes(uint32_t to, uint32_t term, const Ahead<T> &x) {
    uint32_t q[N][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t t[N];
        x.template pair<N>(t, i);
#pragma unroll
        for (int n = 0; n < N; ++n) q[n][i] = t[n];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) tc::tmem_store(to + n * term, q[n]);
}
// A warp has written its left factors: its lane 0 arrives for it.
__device__ __forceinline__ void ready(uint64_t &bar) {
    tc::tmem_stored();
    tc::fence_before_sync();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) tc::bar_arrive(tc::smem_addr(&bar));
}
// Values of row `row` from block `first` on as float32 blocks, `width` blocks a row.
template <int N>
__device__ __forceinline__ void keep_row(uint8_t *to, int row, int width, int first, const float (&v)[N]) {
    to += (uint32_t)((row / 8 * width + first) * kWide + (row & 7) * 32);
#pragma unroll
    for (int n = 0; n < N / 8; ++n) {
        uint32_t q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = __float_as_uint(v[n * 8 + e]);
        tc::store32(to + n * kWide, q);
    }
}
// A thread's tokens of a column as tiles of bfloat16 terms [term][columns of 8][tokens of 8].
template <int NT, typename T>
__device__ __forceinline__ void keep_values(uint8_t *to, uint32_t term, int row, int first, const Ahead<T> &x) {
    to += (uint32_t)((row / 8 * 8 + first) * kCell + (row & 7) * 16);
#pragma unroll
    for (int n = 0; n < kTokens / 8; ++n) {
        uint32_t q[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i) x.template pair<NT>(q[i], n * 4 + i);
#pragma unroll
        for (int m = 0; m < NT; ++m) *reinterpret_cast<uint4 *>(to + m * term + n * kCell) = make_uint4(q[0][m], q[1][m], q[2][m], q[3][m]);
    }
}

struct Bars {
    uint64_t tiles[2], free[2];            // a stage's tiles have come; all that reads them is done
    uint64_t first, second, third;         // all warps have written a round's left factors
    uint64_t one, two, three, four;        // products are done
};
struct Waits {
    bool ok;
    __device__ __forceinline__ void operator()(uint64_t &bar, uint32_t phase) { ok = ok && tc::bar_wait(tc::smem_addr(&bar), phase & 1); }
    __device__ __forceinline__ bool all() { return ok = __all_sync(0xffffffffu, ok); }     // of a warp's lanes
    // of products: what they wrote may be read then
    __device__ __forceinline__ void done(uint64_t &bar, uint32_t phase) {
        operator()(bar, phase);
        tc::fence_after_sync();
    }
};

// 96 registers a thread at the launch (the compiler's choice for 640 threads), 104 and 64 after: as many in all.
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 104;"); }
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 64;"); }
// What both walks begin and end with.
__device__ __forceinline__ uint32_t begin(Bars &bars, uint32_t &where, int warps) {
    if (threadIdx.x == 0) {
        uint64_t *all[] = {&bars.tiles[0], &bars.tiles[1], &bars.free[0], &bars.free[1], &bars.one, &bars.two, &bars.three, &bars.four};
        for (uint64_t *b : all) tc::bar_init(tc::smem_addr(b), 1);
        tc::bar_init(tc::smem_addr(&bars.first), warps);
        tc::bar_init(tc::smem_addr(&bars.second), warps);
        tc::bar_init(tc::smem_addr(&bars.third), warps);
        tc::bar_init_fence();
    }
    if (threadIdx.x < 32) tc::tmem_alloc_one(tc::smem_addr(&where), kColumns);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    return __shfl_sync(0xffffffffu, where, 0);
}
__device__ __forceinline__ void finish(bool ok, uint32_t tmem) {
    if (!ok) let_land();
    tc::fence_before_sync();
    __syncthreads();
    if (threadIdx.x < 32) tc::tmem_free_one(tmem, kColumns);
}

// Columns of tensor memory, forward: the state's terms, then those of rest u | k S and q S, then the state's change |
// terms of v - first k S, then of u | e, then P u.
constexpr uint32_t kState = 0, kSeen = 192, kError = 320, kOut = 416;

template <typename T, int DKP, bool KEEP>
__global__ void __launch_bounds__(kThreads, 1) delta_forward_kernel(const __grid_constant__ Args a, const T *v, const float *s0, T *o, float *last,
                                                                    uint8_t *kept, int stages, int columns) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3, W = DKP / 8, TILE = 64 * DKP * 2, SQ = kSquare / 3, OWN = DKP / kParts;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Bars bars;
    __shared__ uint32_t where;
    pdl_begin();
    const int b = blockIdx.x / a.Hv, h = blockIdx.x % a.Hv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), part = warp >> 2;
    const int in = (warp & 3) * 32 + (threadIdx.x & 31), col = blockIdx.y * columns + in, tok0 = part * kTokens;
    const Sequence s = sequence(a, b);
    const int chunks = (s.length + C - 1) / C;
    const Stage st = stage_of(a.p);
    const bool here = col < a.Dv, kept_here = KEEP && col < a.p.DVP;
    const int64_t state = ((int64_t)b * a.Hv + h) * a.Dk * a.Dv, stride = s.step * a.Hv * a.Dv;
    const int64_t first = ((s.row + tok0 * s.step) * a.Hv + h) * a.Dv + col;
    const uint32_t base = tc::smem_addr(smem), tmem = begin(bars, where, kParts * (columns / 32));
    const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21);          // this warp's lanes
    Waits wait{true};
    if (warp >= kWarps) {
        fewer_registers();
        if (warp == kWarps + 1)
            for (int n = 0; n < chunks; ++n) {
                const int at = stage_at(n, stages);
                if (n >= stages) wait(bars.free[at], free_phase(n, stages));
                if (!wait.all()) break;
                load_stage(a, st, base + at * st.bytes, tc::smem_addr(&bars.tiles[at]), kept, a.p.xe, s.slot + n, h);
            }
        if (warp == kWarps && tc::elected()) {
            for (int n = 0; n < chunks && wait.ok; ++n) {
                const int at = stage_at(n, stages);
                const uint32_t tiles = base + at * st.bytes, k = tiles + st.k, q = tiles + st.q, x = tiles + st.x, p = tiles + st.p;
                wait(bars.tiles[at], n / stages);
                wait.done(bars.first, n);
                if (!wait.ok) break;
                tc::issue<3, NT, 3, DKP / 16, 64, W, false, 0>(tmem + kSeen, tmem + kState, DKP / 2, k, TILE);
                tc::commit_one(tc::smem_addr(&bars.one));
                tc::issue<3, NT, 3, DKP / 16, 64, W, false, 0>(tmem + kSeen + 64, tmem + kState, DKP / 2, q, TILE);
                wait.done(bars.second, n);
                if (!wait.ok) break;
                tc::issue<3, 3, 3, 4, 64, 8, false, 1>(tmem + kOut, tmem + kError, 32, x, SQ);
                tc::commit_one(tc::smem_addr(&bars.two));
                wait.done(bars.third, n);
                if (!wait.ok) break;
                tc::issue<3, NT, 3, 4, DKP, W, true, 0>(tmem + kSeen, tmem + kState, 32, k, TILE);
                tc::commit_one(tc::smem_addr(&bars.three));
                tc::issue<3, 3, 3, 4, 64, 8, false, 1>(tmem + kOut, tmem + kError, 32, p, SQ);
                tc::commit_one(tc::smem_addr(&bars.four));
                tc::commit_one(tc::smem_addr(&bars.free[at]));
            }
        }
        __syncwarp();
        finish(wait.ok, tmem);
        return;
    }
    more_registers();
    if ((warp & 3) * 32 >= columns) {      // lanes without a column
        finish(wait.ok, tmem);
        return;
    }
    float S[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int d = part * OWN + i;
        S[i] = s0 && here && d < a.Dk ? s0[state + (int64_t)d * a.Dv + col] : 0.f;
    }
    Ahead<T> ahead;
    fetch(ahead, v + first, stride, here ? s.length - tok0 : 0);
    float out[kTokens];
    auto put_out = [&](int n) {        // o of chunk n: what of it lies in registers and P u
        wait.done(bars.four, n);
        float u[kTokens];
        tc::tmem_load(u, mine + kOut + tok0);
#pragma unroll
        for (int i = 0; i < kTokens; ++i) u[i] = a.scale * (out[i] + u[i]);
        if (!wait.ok)
#pragma unroll
            for (int i = 0; i < kTokens; ++i) u[i] = __int_as_float(0x7fffffff);
        T *to = o + first + (int64_t)n * C * stride;
        const int left = here ? s.length - n * C - tok0 : 0;
        if (left >= kTokens) {
#pragma unroll
            for (int i = 0; i < kTokens; ++i, to += stride) put(to, u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kTokens; ++i, to += stride)
                if (i < left) put(to, u[i]);
        }
    };
    for (int n = 0; n < chunks; ++n) {
        const int at = stage_at(n, stages);
        const int64_t hv = (s.slot + n) * a.Hv + h;
        to_lanes<3>(mine + kState + part * (OWN / 2), DKP / 2, S);
        ready(bars.first);
        if (n) put_out(n - 1);
        // what the backward needs goes out a little in each round: an SM's stores take 64 bytes a cycle at best
        if (kept_here) keep_values<NT>(kept + a.p.v + hv * a.p.value_bytes, (uint32_t)(C * a.p.DVP * 2), col, part * (kTokens / 8), ahead);
        wait(bars.tiles[at], n / stages);
        const float *gates = reinterpret_cast<const float *>(smem + at * st.bytes + st.gates);
        const float keep = gates[kKeep];
        float r[kTokens];
        wait.done(bars.one, n);
        tc::tmem_load(r, mine + kSeen + tok0);
        each(gates + kFirst + tok0, [&](int i, float f) { r[i] = fmaf(-f, r[i], ahead.get(i)); });
        to_lanes<3>(mine + kError + part * (kTokens / 2), 32, r);
        ready(bars.second);
        fetch(ahead, v + first + (int64_t)(n + 1) * C * stride, stride, here ? s.length - (n + 1) * C - tok0 : 0);
        if (kept_here) keep_row(kept + a.p.s + hv * a.p.state_bytes, col, W, part * (W / kParts), S);
        wait.done(bars.two, n);
        tc::tmem_load(r, mine + kOut + tok0);
        if (kept_here) keep_row(kept + a.p.e + hv * a.p.kept_bytes, col, 8, part * (kTokens / 8), r);
        each(gates + kBeta + tok0, [&](int i, float g) { r[i] *= g; });
        to_lanes<3>(mine + kError + part * (kTokens / 2), 32, r);
        each(gates + kRest + tok0, [&](int i, float g) { r[i] *= g; });
        to_lanes<3>(mine + kState + part * (kTokens / 2), 32, r);
        tc::tmem_load(out, mine + kSeen + 64 + tok0);
        each(gates + kFirst + tok0, [&](int i, float f) { out[i] *= f; });
        ready(bars.third);
        wait.done(bars.three, n);
#pragma unroll
        for (int w = 0; w < OWN / 16; ++w) {
            float d[16];
            tc::tmem_load(d, mine + kSeen + part * OWN + w * 16);
#pragma unroll
            for (int i = 0; i < 16; ++i) S[w * 16 + i] = fmaf(keep, S[w * 16 + i], d[i]);
        }
        if (!wait.ok)
#pragma unroll
            for (int i = 0; i < OWN; ++i) S[i] = __int_as_float(0x7fffffff);
    }
    if (chunks) put_out(chunks - 1);
    if (kept_here) keep_row(kept + a.p.end + ((int64_t)b * a.Hv + h) * a.p.state_bytes, col, W, part * (W / kParts), S);
    if (last && here)
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int d = part * OWN + i;
            if (d < a.Dk) last[state + (int64_t)d * a.Dv + col] = S[i];
        }
    finish(wait.ok, tmem);
}

// Columns of tensor memory, backward: terms of the state's gradient, then (from the same place) those of scale first
// go | those of go | of d, then of -first b y | k D, then y | P^T go. The change of the state's gradient: q's part in
// the place of its terms' last third and of go's terms, k's where y and P^T go were, when these are done with.
// (Two sums: the matrix instruction cuts off where it should round, a little more with every 16 summed places.)
constexpr uint32_t kGrad = 0, kGo = 192, kD = 288, kY = 384, kPg = 448, kChange = 96;

template <typename T, int DKP>
__global__ void __launch_bounds__(kThreads, 1) delta_backward_kernel(const __grid_constant__ Args a, const T *go, const uint8_t *kept, uint8_t *scratch,
                                                                     const float *glast, float *gs0, int stages, int columns) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3, W = DKP / 8, TILE = 64 * DKP * 2, SQ = kSquare / 3, OWN = DKP / kParts;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Bars bars;
    __shared__ uint32_t where;
    pdl_begin();
    const int b = blockIdx.x / a.Hv, h = blockIdx.x % a.Hv, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), part = warp >> 2;
    const int in = (warp & 3) * 32 + (threadIdx.x & 31), col = blockIdx.y * columns + in, tok0 = part * kTokens;
    const Sequence s = sequence(a, b);
    const int chunks = (s.length + C - 1) / C;
    const Stage st = stage_of(a.p);
    const bool here = col < a.Dv, kept_here = col < a.p.DVP;
    const int64_t state = ((int64_t)b * a.Hv + h) * a.Dk * a.Dv, stride = s.step * a.Hv * a.Dv;
    const int64_t first = ((s.row + tok0 * s.step) * a.Hv + h) * a.Dv + col;
    const uint32_t base = tc::smem_addr(smem), tmem = begin(bars, where, kParts * (columns / 32));
    const uint32_t mine = tmem + ((uint32_t)(warp & 3) << 21);
    Waits wait{true};
    if (warp >= kWarps) {
        fewer_registers();
        if (warp == kWarps + 1)
            for (int n = 0; n < chunks; ++n) {
                const int at = stage_at(n, stages);
                if (n >= stages) wait(bars.free[at], free_phase(n, stages));
                if (!wait.all()) break;
                load_stage(a, st, base + at * st.bytes, tc::smem_addr(&bars.tiles[at]), kept, a.p.xu, s.slot + chunks - 1 - n, h);
            }
        if (warp == kWarps && tc::elected()) {
            for (int n = 0; n < chunks; ++n) {
                const int at = stage_at(n, stages);
                const uint32_t tiles = base + at * st.bytes, k = tiles + st.k, q = tiles + st.q, x = tiles + st.x, p = tiles + st.p;
                wait(bars.tiles[at], n / stages);
                wait.done(bars.first, n);
                if (!wait.ok) break;
                tc::issue<3, NT, 3, DKP / 16, 64, W, false, 0>(tmem + kY, tmem + kGrad, DKP / 2, k, TILE);
                tc::issue<NT, 3, 3, 4, 64, 8, true, 2>(tmem + kPg, tmem + kGo, 32, p, SQ);
                tc::commit_one(tc::smem_addr(&bars.one));
                wait.done(bars.second, n);
                if (!wait.ok) break;
                tc::issue<3, 3, 3, 4, 64, 8, true, 2>(tmem + kY, tmem + kD, 32, x, SQ);
                tc::commit_one(tc::smem_addr(&bars.two));
                tc::issue<3, NT, 3, 4, DKP, W, true, 0>(tmem + kChange, tmem + kGrad, 32, q, TILE);
                wait.done(bars.third, n);
                if (!wait.ok) break;
                tc::issue<3, NT, 3, 4, DKP, W, true, 0>(tmem + kY, tmem + kD, 32, k, TILE);
                tc::commit_one(tc::smem_addr(&bars.three));
                tc::commit_one(tc::smem_addr(&bars.free[at]));
            }
        }
        __syncwarp();
        finish(wait.ok, tmem);
        return;
    }
    more_registers();
    if ((warp & 3) * 32 >= columns) {      // lanes without a column
        finish(wait.ok, tmem);
        return;
    }
    float D[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int d = part * OWN + i;
        D[i] = glast && here && d < a.Dk ? glast[state + (int64_t)d * a.Dv + col] : 0.f;
    }
    Ahead<T> ahead;
    fetch(ahead, go + first + (int64_t)(chunks - 1) * C * stride, stride, here && chunks ? s.length - (chunks - 1) * C - tok0 : 0);
    for (int n = 0; n < chunks; ++n) {
        const int chunk = chunks - 1 - n, at = stage_at(n, stages);
        const int64_t hv = (s.slot + chunk) * a.Hv + h;
        to_lanes<3>(mine + kGrad + part * (OWN / 2), DKP / 2, D);
        to_lanes<NT>(mine + kGo + part * (kTokens / 2), 32, ahead);
        ready(bars.first);
        if (kept_here) keep_values<NT>(scratch + a.p.go + hv * a.p.value_bytes, (uint32_t)(C * a.p.DVP * 2), col, part * (kTokens / 8), ahead);
        wait(bars.tiles[at], n / stages);
        const float *gates = reinterpret_cast<const float *>(smem + at * st.bytes + st.gates);
        const float keep = gates[kKeep];
        float r[kTokens];
        wait.done(bars.one, n);
        {
            float d[kTokens];
            tc::tmem_load(r, mine + kY + tok0);
            tc::tmem_load(d, mine + kPg + tok0);
            each(gates + kRest + tok0, [&](int i, float g) { r[i] = fmaf(g, r[i], a.scale * d[i]); });
        }
        to_lanes<3>(mine + kD + part * (kTokens / 2), 32, r);
        each(gates + kFirst + tok0, [&](int i, float f) { r[i] = a.scale * f * ahead.get(i); });
        to_lanes<3>(mine + kGrad + part * (kTokens / 2), 32, r);
        ready(bars.second);
        if (n + 1 < chunks) fetch(ahead, go + first + (int64_t)(chunk - 1) * C * stride, stride, here ? kTokens : 0);
        if (kept_here) keep_row(scratch + a.p.d + hv * a.p.state_bytes, col, W, part * (W / kParts), D);
        wait.done(bars.two, n);
        tc::tmem_load(r, mine + kY + tok0);
        if (kept_here) keep_row(scratch + a.p.y + hv * a.p.kept_bytes, col, 8, part * (kTokens / 8), r);
        each(gates + kFirst + tok0, [&](int i, float f) { r[i] *= -f; });
        each(gates + kBeta + tok0, [&](int i, float g) { r[i] *= g; });
        to_lanes<3>(mine + kD + part * (kTokens / 2), 32, r);
        ready(bars.third);
        wait.done(bars.three, n);
#pragma unroll
        for (int w = 0; w < OWN / 16; ++w) {
            float y[16], z[16];
            tc::tmem_load(y, mine + kChange + part * OWN + w * 16);
            tc::tmem_load(z, mine + kY + part * OWN + w * 16);
#pragma unroll
            for (int i = 0; i < 16; ++i) D[w * 16 + i] = fmaf(keep, D[w * 16 + i], y[i] + z[i]);
        }
        if (!wait.ok)
#pragma unroll
            for (int i = 0; i < OWN; ++i) D[i] = __int_as_float(0x7fffffff);
        // the other warps of these lanes have read their parts before terms are written over them
        asm volatile("bar.sync %0, %1;" ::"r"(1 + (warp & 3)), "n"(32 * kParts) : "memory");
    }
    if (gs0 && here)
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int d = part * OWN + i;
            if (d < a.Dk) gs0[state + (int64_t)d * a.Dv + col] = D[i];
        }
    finish(wait.ok, tmem);
}

// Columns of v a block takes: all, or, where there are SMs left over, 32 or 64 of them (columns do not meet; what is
// shared is the tiles' loads and the chain's length). 18 heads of 40 x 72, 509 tokens in float32,
// forward and backward: all columns a block 37.3 and 40.7 us, 32 of them 35.9 and 37.6.
int columns_of(const Args &a) {
    const int64_t heads = (int64_t)a.B * a.Hv;
    const int all = (a.Dv + 31) / 32 * 32;
    for (int columns = 32; columns < all; columns *= 2)
        if (heads * ((all + columns - 1) / columns) <= 152) return columns;
    return all;
}
// One or two stages of shared memory.
int stages_of(const Args &a) { return 2 * stage_of(a.p).bytes <= 225 * 1024 ? 2 : 1; }

template <typename K, typename... A>
cudaError_t walk(K kernel, const Args &a, cudaStream_t s, A... args) {
    const size_t smem = (size_t)stages_of(a) * stage_of(a.p).bytes;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    const int columns = columns_of(a);
    const dim3 grid((unsigned)(a.B * a.Hv), (unsigned)((a.Dv + columns - 1) / columns));
    return e != cudaSuccess ? e : seq_launch(kernel, grid, kThreads, smem, s, 1, a, args..., stages_of(a), columns);
}
template <typename T, int DKP>
cudaError_t forward(const Args &a, const void *v, const float *s0, void *o, float *last, uint8_t *kept, bool keep, cudaStream_t s) {
    return keep ? walk(delta_forward_kernel<T, DKP, true>, a, s, (const T *)v, s0, (T *)o, last, kept)
                : walk(delta_forward_kernel<T, DKP, false>, a, s, (const T *)v, s0, (T *)o, last, kept);
}

}  // namespace
}  // namespace delta

cudaError_t delta_walk_forward(const delta::Args &a, bool bf16, const void *v, const float *s0, void *o, float *last, uint8_t *kept, bool keep,
                               cudaStream_t s) {
    using namespace delta;
    auto go = [&](auto run) { return run(a, v, s0, o, last, kept, keep, s); };
    return bf16 ? (a.p.DKP == 64 ? go(forward<__nv_bfloat16, 64>) : go(forward<__nv_bfloat16, 128>))
                : (a.p.DKP == 64 ? go(forward<float, 64>) : go(forward<float, 128>));
}

cudaError_t delta_walk_backward(const delta::Args &a, bool bf16, const void *go, const float *glast, const uint8_t *kept, uint8_t *scratch,
                                float *gs0, cudaStream_t s) {
    using namespace delta;
    if (bf16) {
        const __nv_bfloat16 *g = static_cast<const __nv_bfloat16 *>(go);
        return a.p.DKP == 64 ? walk(delta_backward_kernel<__nv_bfloat16, 64>, a, s, g, kept, scratch, glast, gs0)
                             : walk(delta_backward_kernel<__nv_bfloat16, 128>, a, s, g, kept, scratch, glast, gs0);
    }
    const float *g = static_cast<const float *>(go);
    return a.p.DKP == 64 ? walk(delta_backward_kernel<float, 64>, a, s, g, kept, scratch, glast, gs0)
                         : walk(delta_backward_kernel<float, 128>, a, s, g, kept, scratch, glast, gs0);
}

}  // namespace dendsn
