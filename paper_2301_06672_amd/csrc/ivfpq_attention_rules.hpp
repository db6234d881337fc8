// How the work of ivfpq_draft_attention is divided, by sizes alone.  Plain C++, so that a test can ask the same rules.
#pragma once

#include <algorithm>
#include <cstdint>

namespace ivfpq {

struct AttentionPlan {
    int tiles;                        // of 16 columns a wave; a column is a row of the pass for one of the heads that share keys
    bool apart;                       // each wave has columns of its own; else the waves share them and divide the places
    int waves;                        // of a workgroup
    int blocks;                       // of columns
    int parts;                        // that the places of all sequences together are dealt to, for each head and block; 0: a workgroup a sequence
    int columns() const { return tiles * 16 * (apart ? waves : 1); }
};

constexpr int kMostPartsEach = 64;    // of a sequence, on average: what is joined one after the other

inline AttentionPlan attention_plan(int64_t n, int m, int heads, int kv_heads, int d, int64_t max_places) {
    const int64_t columns = (int64_t)m * (heads / kv_heads);
    AttentionPlan p{};
    // Waves share up to 32 columns, 16 of long heads, whose sums leave room in the registers for keys and values on their way.  (12 rows of 8 sequences of
    // up to 4,000 places, 32 heads over 8: 48 columns shared 63 us, apart 39; 24 rows of 128 components 62 with two tiles a wave and one block, 55 with one tile and
    // two blocks; of 256 components, 64 rows 254 with two tiles a wave, 158 with one.  8 rows, 32 columns: shared 48 of those and 158 of 32 sequences of up
    // to 8,000 places, apart 38 and 178.)
    p.apart = columns > (d > 128 ? 16 : 32);
    p.waves = p.apart && columns > 128 && d <= 128 ? 8 : 4;
    p.tiles = p.apart ? (p.waves == 8 ? 2 : 1) : columns <= 16 ? 1 : 2;
    p.blocks = (int)((columns + p.columns() - 1) / p.columns());
    // Where sequences are too few to fill the GPU: some 512 parts of all heads and blocks together, of two tiles a wave at least, equal whatever the lengths.  A
    // part that holds the end of a sequence is a piece more, so there are up to (parts + n) * groups.  (Workgroups that a CU has room for, by registers and LDS, of heads
    // of up to 64, up to 128 and more components: shared columns of one tile 3, 2, 1, of two 2, 1; apart with four waves 3, 2, 1, with eight 1.  512 is not fitted to each
    // of them: the 576 pieces of 8 rows of 8 sequences, two tiles shared, 48 us, come in over two rounds of 256; those of 12 rows, apart, 39 us, in one of 512 and a rest.)
    // (One row over 2,049 places, 32 heads of 128 over 8: parts of 128, 256 and 512 places take 10.1, 9.4 and 11.7 us, and joining them 6.5, 5.1 and 4.2.)
    // The kernel of eight waves leaves room for one workgroup on a CU: a part for each of one sequence, and of several, whose pieces differ, two rounds
    // of pieces (64 rows of 16 sequences of 2,111 to 8,191 places, 32 heads of 128 over 8: 384, 512, 640, 768, 1,024 pieces take 181, 161, 162, 170, 174 us,
    // and joining them 13, 16, 18, 22, 28).
    // Where parts would be no more than sequences, from 64 sequences of single tokens and 32 of 64 rows on with 8 heads of keys, a workgroup has a whole sequence.  With
    // lengths from the longest evenly down to a quarter of it nothing is lost: 64 rows of 31, 32 and 33 sequences up to 8,192 places 1.92, 1.64 and 1.79 ns a place,
    // single tokens of 63, 64 and 80 up to 16,384 0.76, 0.77 and 0.78.  One long sequence among short ones is left to its own workgroups there: 65,536 places beside
    // 1,000 each take 179 us with 31 sequences of 64 rows and 1,930 with 32, 120 us with 63 of single tokens and 1,400 with 64.
    const int64_t groups = (int64_t)kv_heads * p.blocks, useful = n * max_places / (p.apart ? 128 : 256);
    const int64_t wanted = p.waves == 8 ? (n == 1 ? (256 + groups - 1) / groups : 512 / groups - n) : (512 + groups - 1) / groups;
    const int64_t parts = std::min<int64_t>({wanted, useful, kMostPartsEach * n});
    p.parts = parts > n ? (int)parts : 0;
    return p;
}

// Whether the tiles of all sequences together, of as many places as the page table has, can be numbered by 31 bits: they are where they are dealt to parts.
inline bool tiles_numbered(int64_t n, int64_t table_places) { return n * (table_places / 32 + 2) < ((int64_t)1 << 31); }

// Scratch of divided places, in bytes: for every head, block and piece (a part's share of a sequence) the sums of d components for each column, then their
// references and sums of weights; then the first and last part of every sequence and block.
inline int64_t attention_pieces(int64_t n, int kv_heads, const AttentionPlan& p) { return p.parts ? (int64_t)kv_heads * p.blocks * (p.parts + n) * p.columns() : 0; }
inline int64_t attention_scratch_bytes(int64_t n, int kv_heads, int d, const AttentionPlan& p) {
    return p.parts ? attention_pieces(n, kv_heads, p) * ((int64_t)d + 2) * 4 + n * p.blocks * 8 : 0;
}

}  // namespace ivfpq
