// How the work of ivfpq_draft_attention is divided, by sizes alone.  Plain C++, so that a test can ask the same rules.
#pragma once

#include <algorithm>
#include <cstdint>

namespace ivfpq {

struct AttentionPlan {
    int tiles;                        // of 16 columns a wave; a column is a row of the pass for one of the heads that share keys
    bool apart;                       // each wave has columns of its own; else the waves share them and divide the places
    int blocks;                       // of columns
    int splits;                       // of the places
    int waves;                        // of a workgroup
    int columns() const { return tiles * 16 * (apart ? waves : 1); }
};

constexpr int kMostSplits = 64;

inline AttentionPlan attention_plan(int64_t n, int m, int heads, int kv_heads, int d, int64_t max_places) {
    const int64_t columns = (int64_t)m * (heads / kv_heads);
    const int most = d > 128 ? 2 : 4;                               // tiles whose sums fit a wave's registers
    AttentionPlan p{};
    p.apart = columns > 16 * most;
    p.tiles = p.apart ? 2 : columns <= 16 ? 1 : columns <= 32 ? 2 : most;
    p.waves = p.apart && columns > 128 && d <= 128 ? 8 : 4;
    p.blocks = (int)((columns + p.columns() - 1) / p.columns());
    // workgroups for every CU twice over, each of at least two tiles of places a wave
    const int64_t groups = n * kv_heads * p.blocks;
    const int64_t useful = max_places / (p.apart ? 128 : 256);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(512 + groups - 1) / groups, useful, kMostSplits}));
    return p;
}

// scratch of split places: for every row, head and split the sums of d components, then the reference and the sum of weights
inline int64_t attention_split_floats(int64_t n, int m, int heads, int d, int splits) {
    return splits == 1 ? 0 : n * m * heads * splits * ((int64_t)d + 2);
}

}  // namespace ivfpq
