// Gated delta rule: a matrix of fast weights for every head that a token's key reads, corrects and
// writes,
//   S_t = a_t S_{t-1} + k_t u_t^T,  u_t = b_t (v_t - a_t S_{t-1}^T k_t),  a_t = exp(gate_t),
//   o_t = scale S_t^T q_t
// and its gradient, in chunks of 64 tokens. Within a chunk, with G_i the sum of the gates up to token i,
// L_ij = exp(G_i - G_j) (k_i . k_j) below the diagonal, P_ij = exp(G_i - G_j) (q_i . k_j) up to it,
// first_i = exp(G_i), rest_i = exp(G_last - G_i) and S the state before the chunk:
//   e  = (1 + L diag(b))^-1 (v - first k S),   u = b e
//   o  = scale (first q S + P u),              S' = exp(G_last) S + k^T (rest u)
// and back, with D the gradient of the state behind the chunk:
//   d  = scale P^T go + rest k D,  y = ((1 + diag(b) L)^-1)^T d,  gv = b y,  gb = e . y
//   D' = exp(G_last) D + q^T (scale first go) - k^T (first b y)
//   gq = scale first go S^T + A k,           A_ij  = scale exp(G_i - G_j) go_i . u_j   (j <= i)
//   gk = rest u D^T - first b y S^T + A^T q + (C + C^T) k, C_ij = -exp(G_i - G_j) b_i y_i . u_j   (j < i)
//   ggate_t = <D, S'> + the sum over i >= t of the chunk of (q_i . gq_i - v_i . gv_i)
// (every exponent in q's gradient raises a product of q, and so on: the sum of what each G_i gains).
//
// What has no order runs for all chunks at once: the square matrices (delta_prepare_kernel), the
// gradients of q, k and the gates (delta_gradients_kernel). In between a block carries the state of one
// head, or the gradient of it, from chunk to chunk (delta_walk.cu).
//
// All sums are float32. Products run on the matrix instruction for 16-bit operands: bfloat16 inputs are
// exact, everything else (float32 inputs, states, results on their way to the next product) is split into
// three bfloat16 terms, whose leading products (three with an exact factor, six without) leave 2^-24.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "delta_common.cuh"
#include "pairs.cuh"
#include "tc_one.cuh"

namespace dendsn {
using namespace delta;
namespace {

// 8 neighbours of a row from `at` on as they lie, zeros behind its end.
template <typename T>
struct Raw {
    uint4 r[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw<T> raw_of(const T *row, int at, int end, bool wide) {
    Raw<T> x;
    if (wide && at + 8 <= end) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) x.r[i] = reinterpret_cast<const uint4 *>(row + at)[i];
    } else {
        uint32_t w[2 * sizeof(T)] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < end) {
                if constexpr (sizeof(T) == 2) w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[at + e] << e % 2 * 16;
                else w[e] = reinterpret_cast<const uint32_t *>(row)[at + e];
            }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) x.r[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
    return x;
}
// Their terms: themselves, or three.
__device__ __forceinline__ void terms_of(uint4 (&t)[1], const Raw<__nv_bfloat16> &x) { t[0] = x.r[0]; }
__device__ __forceinline__ void terms_of(uint4 (&t)[3], const Raw<float> &x) {
    uint32_t q[4][3];
    const uint32_t w[8] = {x.r[0].x, x.r[0].y, x.r[0].z, x.r[0].w, x.r[1].x, x.r[1].y, x.r[1].z, x.r[1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) split<3>(q[i], __uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
#pragma unroll
    for (int n = 0; n < 3; ++n) t[n] = make_uint4(q[0][n], q[1][n], q[2][n], q[3][n]);
}

// ------------------------------------------------------------------ square matrices of a chunk
// exp(G_i - G_j) from the sums in units of log(2), as two floats each, so that far below zero no bits of a difference
// are lost. The hardware's power of two is within 2^-22 of itself.
__device__ __forceinline__ float between(float2 i, float2 j) { return exp2_fast((i.x - j.x) + (i.y - j.y)); }
__device__ __forceinline__ float2 sum_at(const float *gates, int i) { return make_float2(gates[kHigh + i], gates[kLow + i]); }

// Float32 matrices of the chunk in shared memory: rows of 68 floats, so that the pairs a product's registers hold
// are read without bank conflicts.
constexpr int kPitch = 68;
// Left and right factors of 16 x 16 as three terms; `f` gives an element by row and column.
template <typename F>
__device__ __forceinline__ void left_of(uint32_t (&a)[3][4], F f) {
    const int lane = threadIdx.x & 31, g = lane / 4, t = lane % 4 * 2;
    const float lo[4] = {f(g, t), f(g, t + 1), f(g + 8, t), f(g + 8, t + 1)}, hi[4] = {f(g, t + 8), f(g, t + 9), f(g + 8, t + 8), f(g + 8, t + 9)};
    split_left<3>(a, lo, hi);
}
template <typename F>
__device__ __forceinline__ void right_of(uint32_t (&r)[3][4], F f) {
    const int lane = threadIdx.x & 31, g = lane / 4, t = lane % 4 * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = t + (i & 1) * 8, n = g + (i >> 1) * 8;
        uint32_t q[3];
        split<3>(q, f(k, n), f(k + 1, n));
#pragma unroll
        for (int m = 0; m < 3; ++m) r[m][i] = q[m];
    }
}
__device__ __forceinline__ void put_minus(float *x, const float (&r)[2][4]) {
    const int lane = threadIdx.x & 31, g = lane / 4, t = lane % 4 * 2;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        *reinterpret_cast<float2 *>(x + g * kPitch + n * 8 + t) = make_float2(-r[n][0], -r[n][1]);
        *reinterpret_cast<float2 *>(x + (g + 8) * kPitch + n * 8 + t) = make_float2(-r[n][2], -r[n][3]);
    }
}

// One block of 128 threads for a chunk and value head: tiles of k and q (by the first value head of a
// key head), the gates' sums and exponentials, P, and the inverses (1 + L diag(b))^-1 and, for the
// backward, (1 + diag(b) L)^-1: diagonal blocks of 16 by substitution, a thread a column; then twice the corner of
// [[A, 0], [B, D]]^-1 = [[A^-1, 0], [-D^-1 B A^-1, D^-1]], on the matrix instruction. (4096 chunks of 128 places: 136 us,
// 0.4 GB moved; with substitution over all 64 rows 230.)
template <typename T, int DKP, bool KEEP>
__global__ void __launch_bounds__(128) delta_prepare_kernel(const __grid_constant__ Args a, const T *q, const T *k, const float *gate,
                                                            const float *beta, uint8_t *kept, bool wide) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3, W = DKP / 8, TILE = 64 * DKP * 2;
    extern __shared__ __align__(128) uint8_t smem[];
    float *L = reinterpret_cast<float *>(smem);                        // [64][kPitch]
    float *gates = L + 64 * kPitch;
    uint8_t *ktile = reinterpret_cast<uint8_t *>(gates + kGateFloats), *qtile = ktile + NT * TILE;
    float *X = reinterpret_cast<float *>(ktile);                        // [2][64][kPitch], after the products
    pdl_begin();
    int b, chunk;
    Sequence s;
    if (!locate(a, blockIdx.x, &b, &chunk, &s)) return;
    const int h = blockIdx.y, group = a.Hv / a.Hk, hk = h / group, left = min(C, s.length - chunk * C);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane / 4, t = lane % 4;
    const int64_t first = s.row + (int64_t)chunk * C * s.step, head = (int64_t)blockIdx.x * a.Hv + h;
    // 8 places a thread at a time, a tile's loads on their way at once; to the images by the key head's first value head
    const bool leads = h % group == 0;
    auto tile = [&](const T *from, uint8_t *to, uint8_t *image) {
        constexpr int LOTS = C * W / 128;
        Raw<T> r[LOTS];
#pragma unroll
        for (int i = 0; i < LOTS; ++i) {
            const int j = threadIdx.x + i * 128, tok = (j >> 3) / W * 8 + (j & 7);
            r[i] = raw_of(from + ((first + tok * s.step) * a.Hk + hk) * a.Dk, (j >> 3) % W * 8, tok < left ? a.Dk : 0, wide);
        }
#pragma unroll
        for (int i = 0; i < LOTS; ++i) {
            const int at = (threadIdx.x + i * 128) * 16;
            uint4 x[NT];
            terms_of(x, r[i]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                *reinterpret_cast<uint4 *>(to + n * TILE + at) = x[n];
                if (leads) *reinterpret_cast<uint4 *>(image + n * TILE + at) = x[n];
            }
        }
    };
    const int64_t image = ((int64_t)blockIdx.x * a.Hk + hk) * a.p.key_bytes;
    tile(k, ktile, kept + a.p.k + image);
    tile(q, qtile, kept + a.p.q + image);
    if (warp == 0) {           // sums of the gates, in float64: lane l has tokens 2l and 2l + 1
        float r[2], bt[2];
        double sum[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = 2 * lane + e;
            const int64_t at = (first + i * s.step) * a.Hv + h;
            r[e] = i < left ? gate[at] : 0.f;
            bt[e] = i < left ? beta[at] : 0.f;
            if (r[e] < kLeastGate) r[e] = kLeastGate;
        }
        sum[0] = (double)r[0];
        sum[1] = sum[0] + (double)r[1];
        double before = sum[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double up = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += up;
        }
        before -= sum[1];
        const double all = __shfl_sync(0xffffffffu, before + sum[1], 31);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const double G = before + sum[e], units = G * 1.4426950408889634;
            const int i = 2 * lane + e;
            gates[kHigh + i] = (float)units;
            gates[kLow + i] = (float)(units - (double)(float)units);
            gates[kBeta + i] = bt[e];
            gates[kFirst + i] = expf((float)G);
            gates[kRest + i] = expf((float)(all - G));
            gates[kKeep + i] = expf((float)all);
        }
    }
    __syncthreads();
    float *gout = reinterpret_cast<float *>(kept + a.p.gates) + head * kGateFloats;
    for (int i = threadIdx.x; i < kGateFloats; i += 128) gout[i] = gates[i];
    // k k^T and q k^T, 16 rows a warp
    float kk[8][4] = {}, qk[8][4] = {};
    const uint32_t kt = tc::smem_addr(ktile), qt = tc::smem_addr(qtile);
#pragma unroll 2
    for (int ks = 0; ks < W / 2; ++ks) {
        uint32_t ak[NT][4], aq[NT][4], r[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            left_rows(ak[n], kt + n * TILE, W, 2 * warp, 2 * ks);
            left_rows(aq[n], qt + n * TILE, W, 2 * warp, 2 * ks);
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (p > warp) break;
#pragma unroll
            for (int n = 0; n < NT; ++n) right_rows(r[n], kt + n * TILE, W, 2 * p, 2 * ks);
            products<NT, NT, NT>(kk[2 * p], kk[2 * p + 1], ak, r);
            products<NT, NT, NT>(qk[2 * p], qk[2 * p + 1], aq, r);
        }
    }
    uint32_t *pout = reinterpret_cast<uint32_t *>(kept + a.p.p + head * kSquare);
    const float2 Gi[2] = {sum_at(gates, warp * 16 + g), sum_at(gates, warp * 16 + 8 + g)};
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const int j = n * 8 + 2 * t;
        const float2 high = *reinterpret_cast<const float2 *>(gates + kHigh + j), low = *reinterpret_cast<const float2 *>(gates + kLow + j);
        const float2 Gj[2] = {make_float2(high.x, low.x), make_float2(high.y, low.y)};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = warp * 16 + half * 8 + g;
            float w[2] = {}, lo[2] = {};
            if (n < 2 * warp + 2) {        // above the diagonal's blocks there is nothing, and nobody reads
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = between(Gi[half], Gj[e]);
                    w[e] = j + e <= i ? x * qk[n][2 * half + e] : 0.f;
                    lo[e] = j + e < i ? x * kk[n][2 * half + e] : 0.f;
                }
            }
            if (n < 2 * warp + 2) {
                uint32_t x[3];
                split<3>(x, w[0], w[1]);
#pragma unroll
                for (int m = 0; m < 3; ++m) pout[m * 2048 + ((warp * 2 + half) * 8 + n) * 32 + lane] = x[m];
            }
            *reinterpret_cast<float2 *>(L + i * kPitch + j) = make_float2(lo[0], lo[1]);
        }
    }
    __syncthreads();
    const bool back = warp >= 2, mine = KEEP || !back;         // two warps an inverse
    float *x = X + (back ? 64 * kPitch : 0);
    const float *bt = gates + kBeta;
    auto matrix = [&](int i, int j) { return L[i * kPitch + j] * bt[back ? i : j]; };
    if (mine) {
        const int at = (warp & 1) * 32 + (lane & 16), c = lane & 15;
        float z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float d[4] = {};
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const float4 l = *reinterpret_cast<const float4 *>(L + (at + i) * kPitch + at + j);
                d[0] = fmaf(l.x, z[j], d[0]);
                if (j + 1 < i) d[1] = fmaf(l.y, z[j + 1], d[1]);
                if (j + 2 < i) d[2] = fmaf(l.z, z[j + 2], d[2]);
                if (j + 3 < i) d[3] = fmaf(l.w, z[j + 3], d[3]);
            }
            const float sum = (d[0] + d[1]) + (d[2] + d[3]), one = i == c ? 1.f : 0.f, bi = bt[at + i];
            const float r = back ? fmaf(-bi, sum, one) : one - sum;
            z[i] = back ? r : bi * r;
            x[(at + i) * kPitch + at + c] = r;
        }
        __syncwarp();
        // the corner of the warp's 32 rows
        const int r1 = (warp & 1) * 32, r2 = r1 + 16;
        uint32_t l[3][4], r[3][4];
        float u[2][4] = {}, v[2][4] = {};
        left_of(l, [&](int i, int j) { return x[(r2 + i) * kPitch + r2 + j]; });
        right_of(r, [&](int i, int j) { return matrix(r2 + i, r1 + j); });
        products<3, 3, 3>(u[0], u[1], l, r);
        split_left<3>(l, u[0], u[1]);
        right_of(r, [&](int i, int j) { return x[(r1 + i) * kPitch + r1 + j]; });
        products<3, 3, 3>(v[0], v[1], l, r);
        put_minus(x + r2 * kPitch + r1, v);
    }
    __syncthreads();
    if (mine) {        // the corner of all 64: 16 rows a warp
        const int row = 32 + (warp & 1) * 16;
        float u[2][2][4] = {}, v[2][2][4] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k > (warp & 1)) break;
            uint32_t l[3][4], r[3][4];
            left_of(l, [&](int i, int j) { return x[(row + i) * kPitch + 32 + 16 * k + j]; });
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                right_of(r, [&](int i, int j) { return matrix(32 + 16 * k + i, 16 * c + j); });
                products<3, 3, 3>(u[c][0], u[c][1], l, r);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t l[3][4], r[3][4];
            split_left<3>(l, u[k][0], u[k][1]);
#pragma unroll
            for (int c = 0; c <= k; ++c) {
                right_of(r, [&](int i, int j) { return x[(16 * k + i) * kPitch + 16 * c + j]; });
                products<3, 3, 3>(v[c][0], v[c][1], l, r);
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) put_minus(x + row * kPitch + 16 * c, v[c]);
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < (KEEP ? 2 : 1); ++m) {
        uint32_t *out = reinterpret_cast<uint32_t *>(kept + (m ? a.p.xu : a.p.xe) + head * kSquare);
        const float *x = X + m * 64 * kPitch;
#pragma unroll 4
        for (int i = threadIdx.x; i < 2048; i += 128) {
            const int cell = i / 32, row = cell / 8 * 8 + g, col = cell % 8 * 8 + 2 * t;
            if (row / 16 < col / 16) continue;
            const float2 y = *reinterpret_cast<const float2 *>(x + row * kPitch + col);
            uint32_t w[3];
            split<3>(w, y.x, y.y);
#pragma unroll
            for (int n = 0; n < 3; ++n) out[n * 2048 + i] = w[n];
        }
    }
}

// ------------------------------------------------------------------ gradients of q, k and the gates
// Columns of v that a round takes, and places in shared memory. A round's tiles have rows along v: go and y side by
// side (16 blocks a row: both are the left factor of A and C at once), e, the states.
constexpr int kRound = 32;
template <int NT, int DKP>
struct Parts {
    static constexpr uint32_t pair = kRound / 8 * 16 * kCell, error = kRound / 8 * 8 * kCell, state = kRound * DKP * 2;     // bytes of a term
    static constexpr uint32_t t = 0, e = t + 3 * pair, s = e + 3 * error, d = s + 3 * state, rounds = d + 3 * state;
    // where the rounds' tiles were: the square matrices of the chunk, and behind them, of one term, k and q, which come
    // then, so that two blocks share an SM (three terms: beside the tiles, from the start)
    static constexpr bool LATE = NT == 1;
    static constexpr uint32_t a = 0, c = kSquare, key = LATE ? c + kSquare : rounds, keys = NT * C * DKP * 2;
    static_assert(c + kSquare <= key, "what is laid over fits");
    // (64 places: left factors read past their rows)
    static constexpr uint32_t end = (rounds > key + 2 * keys ? rounds : key + 2 * keys) + kCell * 8;
};
// 8 values as bfloat16 terms, 16 bytes each.
template <int N>
__device__ __forceinline__ void put_terms(uint8_t *to, uint32_t term, const float (&v)[8]) {
    uint32_t q[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i) split<N>(q[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int m = 0; m < N; ++m) *reinterpret_cast<uint4 *>(to + m * term) = make_uint4(q[0][m], q[1][m], q[2][m], q[3][m]);
}
__device__ __forceinline__ void floats(float (&v)[8], const uint8_t *from) {
    uint32_t q[8];
    tc::load32(q, from);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(q[i]);
}
// 8 values of NT terms, as they lie in a tile.
template <int NT>
struct Eight {
    uint4 r[NT];
    __device__ __forceinline__ void load(const uint8_t *from, size_t term) {
#pragma unroll
        for (int m = 0; m < NT; ++m) r[m] = *reinterpret_cast<const uint4 *>(from + m * term);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
#pragma unroll
        for (int m = NT - 1; m >= 0; --m) {
            const uint32_t q[4] = {r[m].x, r[m].y, r[m].z, r[m].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] += bf16_low(q[i]), v[2 * i + 1] += bf16_high(q[i]);
        }
    }
};
// Sums over a warp's lanes of 16 values each: lane l returns that of value l / 2.
__device__ __forceinline__ float sums_of(float (&v)[16]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = 8; n; n >>= 1) {
        const bool up = lane & (2 * n);
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + n], 2 * n);
            v[i] = (up ? v[i + n] : v[i]) + other;
        }
    }
    return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

// A block for a chunk and value head. Products with places of Dk as rows (lanes of tensor memory) and tokens as
// columns: S go, S y and D e, over rounds of 32 columns of v, with A and C's sums beside them (rows: tokens of go, of
// y); then those within the chunk. A warp has 8 tokens of a round's go, v, y and e, a lane one column of v. Two blocks
// share an SM (bfloat16), so that one's loads go on beside the other's products. Gradients of shared heads go out in
// float32 for each value head and are added up by delta_join_kernel. (4096 chunks of 128 x 128, bfloat16: 386 us,
// 1.3 GB moved; bound by instructions and latency. In two terms where only gk comes of them 366; with mma.sync, eight warps
// an SM, 760.)
// The matrix instruction cuts its sums off where it should round: every addition onto a large sum costs up to 2^-23 of
// it. So the small products come first, in sums of their own where all of tensor memory is one block's (float32), and
// what is added within the chunk is summed by itself.
// Columns of tensor memory, of the sums through the states and of A and C; those of D e and of A and C are the sums'
// within the chunk afterwards.
constexpr uint32_t kGoS = 0, kYS = 64, kED = 128, kAE = 192, kSums = 256;
template <typename T, int DKP>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) delta_gradients_kernel(const __grid_constant__ Args a, const uint8_t *kept, uint8_t *scratch,
                                                                                       T *gq, T *gk, T *gv, float *ggate, float *gbeta) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3, W = DKP / 8, TILE = C * DKP * 2, SQ = kSquare / 3;
    using P = Parts<NT, DKP>;
    constexpr uint32_t LOW = NT == 1 ? 0 : kSums, kGradColumns = kSums + LOW;      // where the small products' sums are
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t keys_bar, done_bar;
    __shared__ uint32_t where;
    __shared__ __align__(16) float gates[kGateFloats];
    __shared__ float qdot[4][C], edot[C], vdot[C], sums[8];
    pdl_begin();
    int b, chunk;
    Sequence s;
    if (!locate(a, blockIdx.x, &b, &chunk, &s)) return;
    const int h = blockIdx.y, group = a.Hv / a.Hk, lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int64_t hv = (int64_t)blockIdx.x * a.Hv + h, hk = (int64_t)blockIdx.x * a.Hk + h / group;
    const uint32_t base = tc::smem_addr(smem), keys_at = tc::smem_addr(&keys_bar), done = tc::smem_addr(&done_bar);
    if (threadIdx.x == 0) {
        tc::bar_init(keys_at, 1);
        tc::bar_init(done, 1);
        tc::bar_init_fence();
    }
    const uint8_t *kat = kept + a.p.k + hk * a.p.key_bytes, *qat = kept + a.p.q + hk * a.p.key_bytes;
    auto load_keys = [&] {
        if (threadIdx.x) return;
        tc::bar_expect(keys_at, 2 * P::keys);
        load_bytes(base + P::key, kat, P::keys, keys_at);
        load_bytes(base + P::key + P::keys, qat, P::keys, keys_at);
    };
    if (!P::LATE) load_keys();
    if (warp == 0) tc::tmem_alloc_one(tc::smem_addr(&where), kGradColumns);
    const float *gin = reinterpret_cast<const float *>(kept + a.p.gates) + hv * kGateFloats;
    for (int i = threadIdx.x; i < kGateFloats; i += 256) gates[i] = gin[i];
    if (NT == 1)       // go has no second and third term
        for (int i = threadIdx.x; i < 2 * kRound / 8 * 64; i += 256)
            *reinterpret_cast<uint4 *>(smem + P::t + (1 + i / (kRound / 8 * 64)) * P::pair + (i / 64 % (kRound / 8) * 16 * kCell) + i % 64 * 16) = make_uint4(0, 0, 0, 0);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, where, 0);
    const int left = min(C, s.length - chunk * C);
    const int64_t row = s.row + (int64_t)chunk * C * s.step;

    // the state behind the chunk: the next chunk's, or the sequence's last
    const bool ends = (chunk + 1) * C >= s.length;
    const uint8_t *next = ends ? kept + a.p.end + ((int64_t)b * a.Hv + h) * a.p.state_bytes : kept + a.p.s + (hv + a.Hv) * a.p.state_bytes;
    const uint8_t *sat = kept + a.p.s + hv * a.p.state_bytes, *dat = scratch + a.p.d + hv * a.p.state_bytes;
    const uint8_t *yat = scratch + a.p.y + hv * a.p.kept_bytes, *eat = kept + a.p.e + hv * a.p.kept_bytes;
    const uint8_t *goat = scratch + a.p.go + hv * a.p.value_bytes, *vat = kept + a.p.v + hv * a.p.value_bytes;
    const size_t term = (size_t)a.p.DVP * C * 2;
    const int rounds = (a.p.DVP + kRound - 1) / kRound, own = lane / 8 * 8 + warp;     // own: the lane's block of 8 columns and 8 tokens
    float ey[8] = {}, vy[8] = {}, tail = 0.f;
    bool ok = true;            // one value for a warp
    if (threadIdx.x < (P::LATE ? 9 : 7)) {     // all of it is asked for at once, so that the later rounds find it in L2
        const uint8_t *from[] = {sat, dat, next, yat, eat, goat, vat, kat, qat};
        const size_t state = a.p.state_bytes, row_bytes = a.p.kept_bytes, tile = a.p.value_bytes;
        const size_t bytes[] = {state, state, state, row_bytes, row_bytes, tile, tile, P::keys, P::keys};
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from[threadIdx.x]), "r"((uint32_t)bytes[threadIdx.x]) : "memory");
    }
    for (int n = 0; n < rounds; ++n) {
        const int count = min(kRound, a.p.DVP - n * kRound);
        const bool here = lane < count;
        constexpr int LOTS = kRound * W / 256;             // 8 places of a state each
        float y[8] = {}, e[8] = {};
        Eight<NT> go, v;
        if (here) {
            const size_t cell = (size_t)n * kRound + own;
            floats(y, yat + cell * kWide + (lane & 7) * 32);
            floats(e, eat + cell * kWide + (lane & 7) * 32);
            go.load(goat + cell * kCell + (lane & 7) * 16, term);
            v.load(vat + cell * kCell + (lane & 7) * 16, term);
        }
        float S[LOTS][8], D[LOTS][8], behind[LOTS][8];
#pragma unroll
        for (int i = 0; i < LOTS; ++i) {
            const int lot = threadIdx.x + i * 256;
            if (lot < count * W) {
                const size_t at = (size_t)n * kRound * W * 32 + lot * 32;
                floats(S[i], sat + at);
                floats(D[i], dat + at);
                floats(behind[i], next + at);
            }
        }
        if (n) ok = tc::warp_wait(ok, done, (n - 1) & 1);     // the last round's products have read their tiles
        if (here) {
            uint8_t *to = smem + P::t + (lane / 8 * 16 + warp) * kCell + (lane & 7) * 16;
#pragma unroll
            for (int m = 0; m < NT; ++m) *reinterpret_cast<uint4 *>(to + m * P::pair) = go.r[m];
            put_terms<3>(to + 8 * kCell, P::pair, y);
            put_terms<3>(smem + P::e + own * kCell + (lane & 7) * 16, P::error, e);
            float x[8];
            v.get(x);
            const int col = n * kRound + lane, tok0 = warp * 8;
            T *to_v = gv + ((row + tok0 * s.step) * a.Hv + h) * a.Dv + col;
#pragma unroll
            for (int i = 0; i < 8; ++i, to_v += s.step * a.Hv * a.Dv) {
                ey[i] = fmaf(e[i], y[i], ey[i]);
                vy[i] = fmaf(x[i], y[i], vy[i]);
                if (col < a.Dv && tok0 + i < left) put(to_v, gates[kBeta + tok0 + i] * y[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < LOTS; ++i) {
            const int lot = threadIdx.x + i * 256;
            if (lot < count * W) {
                put_terms<3>(smem + P::s + lot * 16, P::state, S[i]);
                put_terms<3>(smem + P::d + lot * 16, P::state, D[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) tail = fmaf(behind[i][j], D[i][j], tail);
            }
        }
        tc::fence_tiles();
        __syncthreads();
        if (warp == (n & 7) && ok && tc::elected()) {      // in turn: issuing takes a warp's time
            tc::fence_after_sync();
            const int steps = count / 16;
            const uint32_t go_at = base + P::t, y_at = go_at + 8 * kCell;
            const bool more = n, after = LOW ? more : true;
            tc::issue_tiles<3, NT, 1, 3, W, 16, true, 0>(tmem + LOW + kGoS, base + P::s, P::state, go_at, P::pair, steps, more);
            tc::issue_tiles<3, NT, 0, 1, W, 16, true, 0>(tmem + kGoS, base + P::s, P::state, go_at, P::pair, steps, after);
            tc::issue_tiles<3, 3, 1, 3, W, 16, true, 0>(tmem + LOW + kYS, base + P::s, P::state, y_at, P::pair, steps, more);
            tc::issue_tiles<3, 3, 0, 1, W, 16, true, 0>(tmem + kYS, base + P::s, P::state, y_at, P::pair, steps, after);
            tc::issue_tiles<3, 3, 1, 3, W, 8, true, 0>(tmem + LOW + kED, base + P::d, P::state, base + P::e, P::error, steps, more);
            tc::issue_tiles<3, 3, 0, 1, W, 8, true, 0>(tmem + kED, base + P::d, P::state, base + P::e, P::error, steps, after);
            tc::issue_tiles<3, 3, 1, 3, 16, 8, true, 0>(tmem + LOW + kAE, go_at, P::pair, base + P::e, P::error, steps, more);
            tc::issue_tiles<3, 3, 0, 1, 16, 8, true, 0>(tmem + kAE, go_at, P::pair, base + P::e, P::error, steps, after);
            tc::commit_one(done);
        }
        __syncwarp();
    }
    {      // e . y and v . y: over the columns, which are the lanes
        float x[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = ey[i], x[8 + i] = vy[i] * gates[kBeta + warp * 8 + i];
        const float dot = sums_of(x);
        if (!(lane & 1)) (lane < 16 ? edot : vdot)[warp * 8 + (lane / 2 & 7)] = dot;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) tail += __shfl_xor_sync(0xffffffffu, tail, o);
    if (lane == 0) sums[warp] = tail;

    ok = tc::warp_wait(ok, done, (rounds - 1) & 1);
    tc::fence_after_sync();
    if (P::LATE && ok) load_keys();
    const int quarter = warp & 3, half = warp >> 2;
    const uint32_t mine = tmem + ((uint32_t)quarter << 21);
    auto sum_load = [&](float (&x)[16], uint32_t from) {
        tc::tmem_load(x, from);
        if (LOW) {
            float low[16];
            tc::tmem_load(low, from + LOW);
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] += low[j];
        }
    };
    // the square matrices as terms: rows 0 to 63 of the sums are A's, the others C's
    const int i = (quarter & 1) * 32 + lane;
    const bool isc = quarter >= 2;
    const float2 Gi = sum_at(gates, i);
    const float mul = isc ? -gates[kBeta + i] : a.scale;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const int j0 = half * 32 + part * 16;
        float x[16];
        sum_load(x, mine + kAE + j0);
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            const float4 high = *reinterpret_cast<const float4 *>(gates + kHigh + j0 + j), low = *reinterpret_cast<const float4 *>(gates + kLow + j0 + j),
                         bt = *reinterpret_cast<const float4 *>(gates + kBeta + j0 + j);
            const float2 Gj[4] = {make_float2(high.x, low.x), make_float2(high.y, low.y), make_float2(high.z, low.z), make_float2(high.w, low.w)};
            const float bj[4] = {bt.x, bt.y, bt.z, bt.w};
            const int end = i - j0 - j + (isc ? 0 : 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j + e] = e < end ? between(Gi, Gj[e]) * (mul * bj[e]) * x[j + e] : 0.f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint8_t *to = smem + (isc ? P::c : P::a) + (i / 8 * 8 + j0 / 8 + c) * kCell + (i & 7) * 16;
            const float z[8] = {x[8 * c], x[8 * c + 1], x[8 * c + 2], x[8 * c + 3], x[8 * c + 4], x[8 * c + 5], x[8 * c + 6], x[8 * c + 7]};
            put_terms<3>(to, SQ, z);
        }
    }
    // what has come through the states, scaled, in place
    if (quarter * 32 < DKP)
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int j0 = half * 32 + part * 16;
            float x[16], z[16];
            sum_load(x, mine + kGoS + j0);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(gates + kFirst + j0 + j);
                x[j] *= a.scale * f.x, x[j + 1] *= a.scale * f.y, x[j + 2] *= a.scale * f.z, x[j + 3] *= a.scale * f.w;
            }
            tc::tmem_put(mine + kGoS + j0, x);
            sum_load(x, mine + kYS + j0);
            sum_load(z, mine + kED + j0);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(gates + kFirst + j0 + j), r = *reinterpret_cast<const float4 *>(gates + kRest + j0 + j),
                             bt = *reinterpret_cast<const float4 *>(gates + kBeta + j0 + j);
                x[j] = bt.x * fmaf(-f.x, x[j], r.x * z[j]);
                x[j + 1] = bt.y * fmaf(-f.y, x[j + 1], r.y * z[j + 1]);
                x[j + 2] = bt.z * fmaf(-f.z, x[j + 2], r.z * z[j + 2]);
                x[j + 3] = bt.w * fmaf(-f.w, x[j + 3], r.w * z[j + 3]);
            }
            tc::tmem_put(mine + kYS + j0, x);
        }
    tc::tmem_stored();
    tc::fence_tiles();
    tc::fence_before_sync();
    __syncthreads();
    ok = tc::warp_wait(ok, keys_at, 0);
    if (warp == 0 && ok && tc::elected()) {
        tc::fence_after_sync();
        const uint32_t k = base + P::key, q = k + P::keys;
        const bool after = !LOW;
        tc::issue_tiles<NT, 3, 1, 3, W, 8, false, 1>(tmem + LOW + kAE, k, TILE, base + P::a, SQ, 4, false);
        tc::issue_tiles<NT, 3, 0, 1, W, 8, false, 1>(tmem + kAE, k, TILE, base + P::a, SQ, 4, after);
        tc::issue_tiles<NT, 3, 1, 3, W, 8, true, 2>(tmem + LOW + kED, q, TILE, base + P::a, SQ, 4, false);
        tc::issue_tiles<NT, 3, 1, 3, W, 8, false, 1>(tmem + LOW + kED, k, TILE, base + P::c, SQ, 4, true);
        tc::issue_tiles<NT, 3, 1, 3, W, 8, true, 2>(tmem + LOW + kED, k, TILE, base + P::c, SQ, 4, true);
        tc::issue_tiles<NT, 3, 0, 1, W, 8, true, 2>(tmem + kED, q, TILE, base + P::a, SQ, 4, after);
        tc::issue_tiles<NT, 3, 0, 1, W, 8, false, 1>(tmem + kED, k, TILE, base + P::c, SQ, 4, true);
        tc::issue_tiles<NT, 3, 0, 1, W, 8, true, 2>(tmem + kED, k, TILE, base + P::c, SQ, 4, true);
        tc::commit_one(done);
    }
    __syncwarp();
    ok = tc::warp_wait(ok, done, rounds & 1);
    tc::fence_after_sync();
    const int d = quarter * 32 + lane;
    const uint8_t *qm = smem + P::key + P::keys + d / 8 * kCell + (d & 7) * 2;
    float *parts = reinterpret_cast<float *>(scratch + a.p.parts);
    if (quarter * 32 < DKP)
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int j0 = half * 32 + part * 16;
            const int64_t tok = row + j0 * s.step;
            float x[16], z[16];
            {
                float add[16];
                tc::tmem_load(x, mine + kGoS + j0);
                sum_load(add, mine + kAE + j0);
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] += add[j];
                tc::tmem_load(z, mine + kYS + j0);
                sum_load(add, mine + kED + j0);
#pragma unroll
                for (int j = 0; j < 16; ++j) z[j] += add[j];
            }
            if (!ok)
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = z[j] = __int_as_float(0x7fffffff);
            auto out = [&](auto *tq, auto *tk, int64_t stride) {
                if (j0 + 16 <= left) {
#pragma unroll
                    for (int j = 0; j < 16; ++j, tq += stride, tk += stride) put(tq, x[j]), put(tk, z[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j, tq += stride, tk += stride)
                        if (j0 + j < left) put(tq, x[j]), put(tk, z[j]);
                }
            };
            if (d < a.Dk) {
                if (group == 1) out(gq + (tok * a.Hk + h) * a.Dk + d, gk + (tok * a.Hk + h) * a.Dk + d, s.step * a.Hk * a.Dk);
                else out(parts + (tok * a.Hv + h) * a.Dk + d, parts + ((a.p.tokens + tok) * a.Hv + h) * a.Dk + d, s.step * a.Hv * a.Dk);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                float v = 0.f;
#pragma unroll
                for (int m = NT - 1; m >= 0; --m)
                    v += value(reinterpret_cast<const __nv_bfloat16 *>(qm + m * TILE + ((j0 + j) / 8 * W) * kCell + ((j0 + j) & 7) * 16));
                x[j] *= v;
            }
            const float dot = sums_of(x);
            if (!(lane & 1)) qdot[quarter][j0 + lane / 2] = dot;
        }
    else
        qdot[quarter][half * 32 + lane] = 0.f;
    if (!ok) let_land();
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_free_one(tmem, kGradColumns);
    if (warp) return;
    // the gates: sums from each token to the chunk's end, and what comes back through the state
    double behind_all = 0.0, at[2];
    for (int w = 0; w < 8; ++w) behind_all += (double)sums[w];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int j = 2 * lane + e;
        at[e] = ((double)qdot[0][j] + (double)qdot[1][j]) + ((double)qdot[2][j] + (double)qdot[3][j]) - (double)vdot[j];
    }
    double behind = at[0] + at[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double down = __shfl_down_sync(0xffffffffu, behind, o);
        if (lane + o < 32) behind += down;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int j = 2 * lane + e;
        if (j >= left) continue;
        const int64_t to = (row + j * s.step) * a.Hv + h;
        // a decay that is 0 in float32 (2^-150) has no gradient
        const float gate = gates[kHigh + j] - (j ? gates[kHigh + j - 1] : 0.f) + (gates[kLow + j] - (j ? gates[kLow + j - 1] : 0.f));
        ggate[to] = gate < -150.f ? 0.f : (float)(behind_all + behind - (e ? at[0] : 0.0));
        gbeta[to] = edot[j];
    }
}

// Gradients of a key head: those of its value heads added up in order, VEC neighbours a thread. blockIdx.y:
// of q, of k. `width`: vectors of a token.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) delta_join_kernel(const __grid_constant__ Args a, const float *parts, T *gq, T *gk, uint32_t width) {
    pdl_begin();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / width;
    if (row >= a.p.tokens) return;
    if (a.layout == DENDSN_DELTA_PACKED && (row < a.offsets[0] || row >= a.offsets[a.B])) return;
    const int at = (int)(i - row * width) * VEC, h = at / a.Dk, d = at - h * a.Dk, group = a.Hv / a.Hk;
    const float *from = parts + ((blockIdx.y * a.p.tokens + row) * a.Hv + (int64_t)h * group) * a.Dk + d;
    float v[VEC] = {};
    for (int j = 0; j < group; ++j) {
        if constexpr (VEC == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(from + (int64_t)j * a.Dk);
            v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        } else {
            v[0] += from[(int64_t)j * a.Dk];
        }
    }
    T *to = (blockIdx.y ? gk : gq) + i * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) put(to + e, v[e]);
}

// Rows of no sequence, as zeros.
struct Rest {
    uint8_t *to[5];
    int64_t bytes[5];          // of a row
};
__global__ void __launch_bounds__(256) delta_rest_kernel(const __grid_constant__ Args a, const __grid_constant__ Rest r) {
    pdl_begin();
    const int64_t lo = min(max(a.offsets[0], 0), a.T), hi = min(max(a.offsets[a.B], 0), a.T), step = (int64_t)gridDim.x * 256;
    for (int n = 0; n < 5; ++n) {
        if (!r.to[n]) continue;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < lo * r.bytes[n] / 2; i += step) reinterpret_cast<uint16_t *>(r.to[n])[i] = 0;
        for (int64_t i = hi * r.bytes[n] / 2 + (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.T * r.bytes[n] / 2; i += step)
            reinterpret_cast<uint16_t *>(r.to[n])[i] = 0;
    }
}

// ------------------------------------------------------------------ few tokens
// A token at a time, as the formulas are written. Columns of v do not meet: a block has 32 of one head's in
// registers, 32 values a thread, LANES threads a row of VEC columns each. Bound by the state's read and
// write: many small blocks keep loads and stores of different blocks on their way at once (64 sequences of 8
// heads of 128 x 128, one token: a block for all columns 19 us, the state's bytes alone 10).
constexpr int kStepColumns = 32, kStepThreads = 128;
template <typename T, int VEC>
__global__ void __launch_bounds__(kStepThreads, 7) delta_step_kernel(const __grid_constant__ Args a, const T *q, const T *k, const T *v, const float *gate,
                                                                     const float *beta, const float *s0, T *o, float *last) {
    constexpr int LANES = kStepColumns / VEC, PASS = kStepThreads / LANES, ROWS = kDeltaMost / PASS;
    __shared__ float ks[kDeltaMost], qs[kDeltaMost], part[2][kStepThreads / 32][kStepColumns];
    pdl_begin();
    const int b = blockIdx.x / a.Hv, h = blockIdx.x % a.Hv, hk = h / (a.Hv / a.Hk), tid = threadIdx.x;
    const int r0 = tid / LANES, in = tid % LANES * VEC, first = blockIdx.y * kStepColumns, col = first + in;
    const Sequence s = sequence(a, b);
    const int64_t state = ((int64_t)b * a.Hv + h) * a.Dk * a.Dv;
    float S[ROWS][VEC];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = r0 + i * PASS;
#pragma unroll
        for (int e = 0; e < VEC; ++e) S[i][e] = 0.f;
        if (s0 && r < a.Dk && col < a.Dv) {
            const float *from = s0 + state + (int64_t)r * a.Dv + col;
            if constexpr (VEC == 4) {
                const float4 x = *reinterpret_cast<const float4 *>(from);
                S[i][0] = x.x, S[i][1] = x.y, S[i][2] = x.z, S[i][3] = x.w;
            } else {
                S[i][0] = *from;
            }
        }
    }
    // sums over the rows of every column: within a warp, then of the warps
    auto gather = [&](float (&x)[VEC], float (*to)[kStepColumns]) {
#pragma unroll
        for (int w = LANES; w < 32; w <<= 1)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], w);
        if ((tid & 31) < LANES)
#pragma unroll
            for (int e = 0; e < VEC; ++e) to[tid / 32][in + e] = x[e];
        __syncthreads();
    };
    auto total = [&](const float (*from)[kStepColumns], int c) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kStepThreads / 32; ++w) x += from[w][c];
        return x;
    };
    for (int n = 0; n < s.length; ++n) {
        const int64_t tok = s.row + n * s.step;
        if (n) __syncthreads();
        for (int i = tid; i < a.Dk; i += kStepThreads) {
            ks[i] = value(k + (tok * a.Hk + hk) * a.Dk + i);
            qs[i] = value(q + (tok * a.Hk + hk) * a.Dk + i);
        }
        const float decay = expf(gate[tok * a.Hv + h]), bt = beta[tok * a.Hv + h];
        float u[VEC], x[VEC] = {}, z[VEC] = {};
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = col + e < a.Dv ? value(v + (tok * a.Hv + h) * a.Dv + col + e) : 0.f;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = r0 + i * PASS;
            const float kr = r < a.Dk ? ks[r] : 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                S[i][e] *= decay;
                x[e] = fmaf(kr, S[i][e], x[e]);
            }
        }
        gather(x, part[0]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = bt * (u[e] - total(part[0], in + e));
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = r0 + i * PASS;
            const float kr = r < a.Dk ? ks[r] : 0.f, qr = r < a.Dk ? qs[r] : 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                S[i][e] = fmaf(kr, u[e], S[i][e]);
                z[e] = fmaf(qr, S[i][e], z[e]);
            }
        }
        gather(z, part[1]);
        if (tid < kStepColumns && first + tid < a.Dv) put(o + (tok * a.Hv + h) * a.Dv + first + tid, a.scale * total(part[1], tid));
    }
    if (!last) return;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = r0 + i * PASS;
        if (r >= a.Dk || col >= a.Dv) continue;
        float *to = last + state + (int64_t)r * a.Dv + col;
        if constexpr (VEC == 4) *reinterpret_cast<float4 *>(to) = make_float4(S[i][0], S[i][1], S[i][2], S[i][3]);
        else *to = S[i][0];
    }
}

// ------------------------------------------------------------------ host
dendsn_status check(const dendsn_delta_config *c) {
    if (!c) return seq_fail(DENDSN_ERR_INVALID_ARG, "cfg is NULL");
    if (c->T < 0 || c->B < 0 || c->Hk < 1 || c->Hv < 1 || c->Dk < 1 || c->Dv < 1)
        return seq_fail(DENDSN_ERR_INVALID_ARG, "T and B must be >= 0, Hk, Hv, Dk and Dv >= 1");
    if (c->Hv % c->Hk) return seq_fail(DENDSN_ERR_INVALID_ARG, "Hv must be a multiple of Hk");
    if (c->x_dtype != DENDSN_F32 && c->x_dtype != DENDSN_BF16) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown x_dtype");
    if (c->layout < DENDSN_DELTA_TIME || c->layout > DENDSN_DELTA_PACKED) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown layout");
    if (c->rest != DENDSN_REST_KEEP && c->rest != DENDSN_REST_ZERO) return seq_fail(DENDSN_ERR_INVALID_ARG, "unknown rest");
    if (!std::isfinite(c->scale)) return seq_fail(DENDSN_ERR_INVALID_ARG, "scale must be finite");
    if (c->Dk > kDeltaMost || c->Dv > kDeltaMost) return seq_fail(DENDSN_ERR_UNSUPPORTED, "Dk or Dv above %d", kDeltaMost);
    if (c->Hv > 65535) return seq_fail(DENDSN_ERR_UNSUPPORTED, "more than 65535 value heads");
    const int64_t most = INT32_MAX, slots = c->layout == DENDSN_DELTA_PACKED ? (int64_t)c->T / C + c->B : (int64_t)c->B * ((c->T + (int64_t)C - 1) / C);
    if (slots > most || (int64_t)c->B * c->Hv > most) return seq_fail(DENDSN_ERR_UNSUPPORTED, "more than 2^31 chunks or states");
    return DENDSN_OK;
}

Args args_of(const dendsn_delta_config &c, const int32_t *offsets) {
    return {c.T, c.B, c.Hk, c.Hv, c.Dk, c.Dv, c.layout, c.scale, offsets, delta_plan(c, DENDSN_DELTA_PACKED, c.x_dtype == DENDSN_BF16)};
}

template <typename K>
cudaError_t room(K kernel, size_t smem) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
}

// Tokens of a call that the step kernel takes one by one: a token's step is about 1.5 us, a chunk's way
// through the chunked kernels 15 us.
constexpr int kFewTokens = 8;
bool by_steps(const dendsn_delta_config &c, const void *kept) {
    if (kept) return false;
    return c.T <= kFewTokens;
}

template <typename T>
cudaError_t run_step(const Args &a, const void *q, const void *k, const void *v, const float *gate, const float *beta, const float *s0, void *o,
                     float *last, cudaStream_t s) {
    const bool four = a.Dv % 4 == 0 && seq_aligned(s0, 16) && seq_aligned(last, 16);
    const dim3 grid((unsigned)(a.B * a.Hv), (unsigned)((a.Dv + kStepColumns - 1) / kStepColumns));
    return four ? seq_launch(delta_step_kernel<T, 4>, grid, kStepThreads, 0, s, 1, a, (const T *)q, (const T *)k, (const T *)v, gate, beta, s0, (T *)o, last)
                : seq_launch(delta_step_kernel<T, 1>, grid, kStepThreads, 0, s, 1, a, (const T *)q, (const T *)k, (const T *)v, gate, beta, s0, (T *)o, last);
}

template <typename T>
bool wide_of(const void *p, int D) { return seq_aligned(p, 16) && D % (16 / (int)sizeof(T)) == 0; }

template <typename T, int DKP>
cudaError_t run_forward(const Args &a, const void *q, const void *k, const void *v, const float *gate, const float *beta, const float *s0, void *o,
                        float *last, uint8_t *kept, bool keep, cudaStream_t s, int *launches) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3;
    cudaError_t e = cudaSuccess;
    if (a.p.slots) {
        const dim3 grid((unsigned)a.p.slots, (unsigned)a.Hv);
        const bool wide = wide_of<T>(q, a.Dk) && wide_of<T>(k, a.Dk);
        const size_t smem = (64 * kPitch + kGateFloats) * 4 + std::max<size_t>(2 * NT * 64 * DKP * 2, (keep ? 2 : 1) * 64 * kPitch * 4);
        e = keep ? room(delta_prepare_kernel<T, DKP, true>, smem) : room(delta_prepare_kernel<T, DKP, false>, smem);
        if (e == cudaSuccess)
            e = keep ? seq_launch(delta_prepare_kernel<T, DKP, true>, grid, 128, smem, s, 1, a, (const T *)q, (const T *)k, gate, beta, kept, wide)
                     : seq_launch(delta_prepare_kernel<T, DKP, false>, grid, 128, smem, s, 1, a, (const T *)q, (const T *)k, gate, beta, kept, wide);
        ++*launches;
    }
    if (e == cudaSuccess) e = delta_walk_forward(a, NT == 1, v, s0, o, last, kept, keep, s);
    ++*launches;
    return e;
}

template <typename T, int DKP>
cudaError_t run_backward(const Args &a, const void *go, const float *glast, const uint8_t *kept, void *gq, void *gk, void *gv, float *ggate,
                         float *gbeta, float *gs0, uint8_t *scratch, cudaStream_t s, int *launches) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 3;
    const dim3 chunks((unsigned)a.p.slots, (unsigned)a.Hv);
    cudaError_t e = delta_walk_backward(a, NT == 1, go, glast, kept, scratch, gs0, s);
    ++*launches;
    if (!a.p.tokens || e != cudaSuccess) return e;     // (packed sequences have slots without tokens too)
    constexpr size_t smem = Parts<NT, DKP>::end;
    e = room(delta_gradients_kernel<T, DKP>, smem);
    if (e == cudaSuccess)
        e = seq_launch(delta_gradients_kernel<T, DKP>, chunks, 256, smem, s, 1, a, kept, scratch, (T *)gq, (T *)gk, (T *)gv, ggate, gbeta);
    ++*launches;
    if (a.Hv > a.Hk && e == cudaSuccess) {
        const int vec = a.Dk % 4 == 0 ? 4 : 1;
        const int64_t width = (int64_t)a.Hk * a.Dk / vec, n = a.p.tokens * width;
        const dim3 grid((unsigned)((n + 255) / 256), 2);
        const float *parts = (const float *)(scratch + a.p.parts);
        e = vec == 4 ? seq_launch(delta_join_kernel<T, 4>, grid, 256, 0, s, 1, a, parts, (T *)gq, (T *)gk, (uint32_t)width)
                     : seq_launch(delta_join_kernel<T, 1>, grid, 256, 0, s, 1, a, parts, (T *)gq, (T *)gk, (uint32_t)width);
        ++*launches;
    }
    return e;
}

cudaError_t fill_rest(const Args &a, const Rest &r, cudaStream_t s, int *launches) {
    ++*launches;
    return seq_launch(delta_rest_kernel, dim3(152), 256, 0, s, 1, a, r);
}

}  // namespace
}  // namespace dendsn

using namespace dendsn;

extern "C" {

dendsn_status dendsn_delta_workspace_size(const dendsn_delta_config *cfg, size_t *saved_bytes, size_t *forward_bytes, size_t *backward_bytes) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    const DeltaPlan p = delta_plan(*cfg, DENDSN_DELTA_PACKED, cfg->x_dtype == DENDSN_BF16);
    if (saved_bytes) *saved_bytes = p.kept_end;
    if (forward_bytes) *forward_bytes = by_steps(*cfg, nullptr) ? 0 : p.forward_end;
    if (backward_bytes) *backward_bytes = p.backward_end;
    return DENDSN_OK;
}

dendsn_status dendsn_delta_forward(const dendsn_delta_config *cfg, const void *q, const void *k, const void *v, const float *gate,
                                   const float *beta, const int32_t *offsets, const float *s0, void *o, float *last, void *saved,
                                   void *scratch, void *stream) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    const bool packed = cfg->layout == DENDSN_DELTA_PACKED, bf = cfg->x_dtype == DENDSN_BF16;
    const int64_t tokens = packed ? cfg->T : (int64_t)cfg->T * cfg->B;
    if (packed != (offsets != nullptr)) return seq_fail(DENDSN_ERR_INVALID_ARG, "offsets go with the packed layout and no other");
    if (tokens && (!q || !k || !v || !gate || !beta || !o)) return seq_fail(DENDSN_ERR_INVALID_ARG, "q, k, v, gate, beta or o is NULL");
    const size_t sx = bf ? 2 : 4;
    if (!seq_aligned(q, sx) || !seq_aligned(k, sx) || !seq_aligned(v, sx) || !seq_aligned(o, sx) || !seq_aligned(gate, 4) ||
        !seq_aligned(beta, 4) || !seq_aligned(offsets, 4) || !seq_aligned(s0, 4) || !seq_aligned(last, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "q, k, v, gate, beta, offsets, s0, o or last misaligned");
    if (!seq_aligned(saved, 256) || !seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "saved and scratch must be 256-byte aligned");
    const Args a = args_of(*cfg, offsets);
    const bool steps = by_steps(*cfg, saved);
    uint8_t *kept = static_cast<uint8_t *>(saved ? saved : scratch);
    if (!steps && a.p.forward_end && !kept) return seq_fail(DENDSN_ERR_INVALID_ARG, "saved and scratch are both NULL");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int launches = 0;
    cudaError_t e = cudaSuccess;
    if (cfg->B) {
        if (steps) {
            e = bf ? run_step<__nv_bfloat16>(a, q, k, v, gate, beta, s0, o, last, s) : run_step<float>(a, q, k, v, gate, beta, s0, o, last, s);
            ++launches;
        } else {
            auto go = [&](auto run) { return run(a, q, k, v, gate, beta, s0, o, last, kept, saved != nullptr, s, &launches); };
            e = bf ? (a.p.DKP == 64 ? go(run_forward<__nv_bfloat16, 64>) : go(run_forward<__nv_bfloat16, 128>))
                   : (a.p.DKP == 64 ? go(run_forward<float, 64>) : go(run_forward<float, 128>));
        }
    }
    if (e == cudaSuccess && packed && cfg->rest == DENDSN_REST_ZERO && tokens)     // (all of them where there is no sequence)
        e = fill_rest(a, {{static_cast<uint8_t *>(o)}, {(int64_t)sx * cfg->Hv * cfg->Dv}}, s, &launches);
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "delta forward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(launches);
    return DENDSN_OK;
}

dendsn_status dendsn_delta_backward(const dendsn_delta_config *cfg, const void *grad_o, const int32_t *offsets, const float *grad_last,
                                    const void *saved, void *grad_q, void *grad_k, void *grad_v, float *grad_gate, float *grad_beta,
                                    float *grad_s0, void *scratch, void *stream) {
    dendsn_status st = check(cfg);
    if (st != DENDSN_OK) return st;
    const bool packed = cfg->layout == DENDSN_DELTA_PACKED, bf = cfg->x_dtype == DENDSN_BF16;
    const int64_t tokens = packed ? cfg->T : (int64_t)cfg->T * cfg->B;
    if (packed != (offsets != nullptr)) return seq_fail(DENDSN_ERR_INVALID_ARG, "offsets go with the packed layout and no other");
    if (tokens && (!grad_o || !grad_q || !grad_k || !grad_v || !grad_gate || !grad_beta))
        return seq_fail(DENDSN_ERR_INVALID_ARG, "grad_o, grad_q, grad_k, grad_v, grad_gate or grad_beta is NULL");
    const Args a = args_of(*cfg, offsets);
    if (a.p.slots && (!saved || !scratch)) return seq_fail(DENDSN_ERR_INVALID_ARG, "saved or scratch is NULL");
    const size_t sx = bf ? 2 : 4;
    if (!seq_aligned(grad_o, sx) || !seq_aligned(grad_q, sx) || !seq_aligned(grad_k, sx) || !seq_aligned(grad_v, sx) || !seq_aligned(grad_gate, 4) ||
        !seq_aligned(grad_beta, 4) || !seq_aligned(grad_s0, 4) || !seq_aligned(grad_last, 4) || !seq_aligned(offsets, 4))
        return seq_fail(DENDSN_ERR_MISALIGNED, "a gradient or offsets misaligned");
    if (!seq_aligned(saved, 256) || !seq_aligned(scratch, 256)) return seq_fail(DENDSN_ERR_MISALIGNED, "saved and scratch must be 256-byte aligned");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int launches = 0;
    cudaError_t e = cudaSuccess;
    if (cfg->B) {
        auto go = [&](auto run) {
            return run(a, grad_o, grad_last, static_cast<const uint8_t *>(saved), grad_q, grad_k, grad_v, grad_gate, grad_beta, grad_s0,
                       static_cast<uint8_t *>(scratch), s, &launches);
        };
        e = bf ? (a.p.DKP == 64 ? go(run_backward<__nv_bfloat16, 64>) : go(run_backward<__nv_bfloat16, 128>))
               : (a.p.DKP == 64 ? go(run_backward<float, 64>) : go(run_backward<float, 128>));
    }
    if (e == cudaSuccess && packed && cfg->rest == DENDSN_REST_ZERO && tokens) {
        const int64_t nk = (int64_t)sx * cfg->Hk * cfg->Dk, nv = (int64_t)sx * cfg->Hv * cfg->Dv, ng = 4 * (int64_t)cfg->Hv;
        e = fill_rest(a, {{static_cast<uint8_t *>(grad_q), static_cast<uint8_t *>(grad_k), static_cast<uint8_t *>(grad_v),
                           reinterpret_cast<uint8_t *>(grad_gate), reinterpret_cast<uint8_t *>(grad_beta)}, {nk, nk, nv, ng, ng}}, s, &launches);
    }
    if (e != cudaSuccess) return seq_fail(DENDSN_ERR_CUDA, "delta backward launch failed: %s", cudaGetErrorString(e));
    seq_count_launches(launches);
    return DENDSN_OK;
}

}  // extern "C"
