// Sizes and places of the gated delta rule's buffers. Plain C++: no CUDA.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace dendsn {

constexpr int kDeltaChunk = 64;            // tokens of a chunk
constexpr int kDeltaMost = 128;            // largest Dk and Dv
constexpr int kSquare = 3 * 64 * 64 * 2;   // bytes of a chunk's square matrix in three terms
constexpr int kGateFloats = 6 * 64;        // of a chunk and value head: see the kernels

// A stage of shared memory holds chunk n's tiles, then chunk n + stages'. Each stage has a barrier of its own that says
// it is free again, when the last product of the chunk that had it is done: its phase by phase, so that it cannot come
// round a second time while the next tiles are waited for (they are not fetched yet). One barrier for all stages could:
// the other stage's chunk completes it once more, and a wait for a parity then looks like one for what is to come.
constexpr int32_t stage_at(int32_t n, int32_t stages) { return n % stages; }
// What the fetch of chunk n (n >= stages) waits for, of that stage's barrier.
constexpr uint32_t free_phase(int32_t n, int32_t stages) { return (uint32_t)(n / stages - 1); }

// Places in bytes; sizes of one chunk (and head).
struct DeltaPlan {
    int32_t terms;                         // bfloat16 terms of an input
    int32_t DKP, DVP;                      // Dk as the tiles have it (64 or 128), Dv up to a multiple of 16
    int64_t slots;                         // chunks there can be
    int64_t tokens;
    size_t key_bytes, value_bytes, kept_bytes, state_bytes;   // a tile of k or q, of v; e and a state in float32
    // kept: what the backward needs of the forward; without it the forward's scratch starts with the same
    size_t k, q, v, xe, p, gates, forward_end, xu, e, s, end, kept_end;
    // the backward's scratch
    size_t go, y, d, parts, backward_end;
};

template <typename Config>
inline DeltaPlan delta_plan(const Config &c, int layout_packed, bool bf16) {
    DeltaPlan p;
    p.terms = bf16 ? 1 : 3;
    p.DKP = c.Dk <= 64 ? 64 : 128;
    p.DVP = (c.Dv + 15) / 16 * 16;
    const int64_t T = c.T, B = c.B;
    p.slots = c.layout == layout_packed ? T / kDeltaChunk + B : B * ((T + kDeltaChunk - 1) / kDeltaChunk);
    p.tokens = c.layout == layout_packed ? T : T * B;
    p.key_bytes = (size_t)p.terms * 64 * p.DKP * 2;
    p.value_bytes = (size_t)p.terms * 64 * p.DVP * 2;
    p.kept_bytes = (size_t)64 * p.DVP * 4;
    p.state_bytes = (size_t)p.DVP * p.DKP * 4;
    const size_t nk = (size_t)p.slots * c.Hk, nv = (size_t)p.slots * c.Hv;
    size_t at = 0;
    auto take = [&](size_t bytes) { size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    p.k = take(nk * p.key_bytes);
    p.q = take(nk * p.key_bytes);
    p.v = take(nv * p.value_bytes);
    p.xe = take(nv * kSquare);
    p.p = take(nv * kSquare);
    p.gates = take(nv * kGateFloats * 4);
    p.forward_end = at;
    p.xu = take(nv * kSquare);
    p.e = take(nv * p.kept_bytes);
    p.s = take(nv * p.state_bytes);
    p.end = take((size_t)B * c.Hv * p.state_bytes);
    p.kept_end = at;
    at = 0;
    p.go = take(nv * p.value_bytes);
    p.y = take(nv * p.kept_bytes);
    p.d = take(nv * p.state_bytes);
    p.parts = take(c.Hv > c.Hk ? (size_t)2 * p.tokens * c.Hv * c.Dk * 4 : 0);
    p.backward_end = at;
    return p;
}

}  // namespace dendsn
