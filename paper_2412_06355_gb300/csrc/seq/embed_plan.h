// The grid of the embedding gradient's index kernel. Plain C++: no CUDA.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace dendsn {

constexpr int kIndexThreads = 1024;       // of an index block
constexpr int kFewTokens = 8192;          // tokens and rows up to which a cluster forms the index
constexpr int kFewRows = 1 << 18;
constexpr int kMostIndexBlocks = 152;     // one for each SM of a whole GB300; scratch is sized for as many

struct IndexGrid {
    bool cluster;                         // the grid is one cluster
    int32_t blocks, chunk;                // blocks, vocabulary rows of one
};

// A block for every 1024 tokens or 4096 rows, at most a cluster's, or one for each of the device's
// `sms`: the blocks of a cooperative grid have to run at the same time, and a block of 1024 threads
// with the bitmap of positions is alone on its SM.
inline IndexGrid index_grid(int64_t n, int64_t V, int sms) {
    IndexGrid g;
    g.cluster = n <= kFewTokens && V <= kFewRows;
    const int64_t blocks = std::max((n + kIndexThreads - 1) / kIndexThreads, (V + 4 * kIndexThreads - 1) / (4 * kIndexThreads));
    const int64_t most = g.cluster ? 8 : std::max(1, std::min(sms, kMostIndexBlocks));
    g.blocks = (int32_t)std::min(blocks, most);
    while (g.cluster && (g.blocks & (g.blocks - 1))) ++g.blocks;
    g.chunk = (int32_t)((V + g.blocks - 1) / g.blocks);
    return g;
}

}  // namespace dendsn
