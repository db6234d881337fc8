// Attention of drafted rows over a paged cache: ivfpq_draft_attention.
//
// For a row's query q, out = sum_p w_p v_p / sum_p w_p with w_p = 2^(s_p - r), s_p = scale log2(e) q . k_p and any reference r: one pass over the
// places, in which r follows the largest s only when that has left r far behind, and sums so far are scaled then.
//
// The rows of the heads that share keys are columns of two matrix products, S = K Q^T and O = V^T W^T, with 16 x 16 x 32 instructions: a tile is
// 32 places and 16 columns.  Keys are dealt to the rows of the first product so that its results are, lane by lane, the operand of the
// second (place 8 g + j of a tile is with lane group g in both), and the cache holds the values of 8 places side by side, so weights stay where they are
// formed and every operand is read in 16-byte pieces.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_attention_rules.hpp"
#include "ivfpq_cache.hpp"

using namespace ivfpq;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ inline f32x4 multiply(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (std::is_same<T, half_t>::value) {
        typedef half_t v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    } else {
        typedef bf16_t v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
}

// rounded to nearest, ties to even
template <class T>
__device__ inline u32x4 narrow8(const float (&x)[8]) {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (T)x[i];
    return __builtin_bit_cast(u32x4, y);
}

struct AttentionIn {
    const void *q, *k_cache, *v_cache;
    void* out;
    float* lse;                       // [n * m][heads] or null
    float* sums;                      // parts > 0: [kv_heads][blocks][parts + n][cols][d], of part p's share of sequence s in place p + s
    float2* norms;                    // [kv_heads][blocks][parts + n][cols]: reference, sum of weights
    int2* spans;                      // [n][blocks]: the first and the last part that have a share of the sequence
    const int* parents;               // [n][m] or null
    long long q_stride, out_stride, n;
    int heads, blocks, parts, cols;
    float scale;                      // its size, with log2(e): not 0, so that -inf stays what it is
    bool negative;
    Pages at;
};

constexpr int kAttentionThreads = 256, kTile = 32;
// A reference is the largest s of its time less kBelow, and follows when an s is more than kAhead over it: weights are up to 2^14 (fp16 holds
// 65,504), and those under 2^-24 of the largest, which fp16 would cut off, are kept down to 2^-30.
constexpr float kBelow = 6.f, kAhead = 14.f;

// What sums about one reference are multiplied by for a larger one.  Not 0: an infinity among them stays one, and what is under 2^-126 of others is lost
// in them anyway.
__device__ inline float shrink_by(float from, float to) { return from == to || from == -INFINITY ? 1.f : fmaxf(exp2_fast(from - to), 0x1p-126f); }

// What a lane has to know of a column: its row and what that sees of the rows.
__device__ inline uint64_t tree_line(const AttentionIn& in, long long s, int count, int lane) {
    uint64_t line = 0;
    int up = -1;
    if (lane < count) {
        up = in.parents[s * in.at.m + lane];
        if (up < 0 || up >= lane) up = -1;
        line = (uint64_t)1 << lane;
    }
    for (int far = 1; far < 64; far *= 2) {          // a row has up to 63 ancestors
        const uint64_t above = __shfl((unsigned long long)line, max(up, 0));
        const int next = __shfl(up, max(up, 0));
        if (up >= 0) {
            line |= above;
            up = next;
        }
    }
    return line;
}

// The pages of a tile's two halves; -1: not there.  Such a half is read as page 0 (there is one: without pages there are no tiles), and the tile is gone
// over with a mask.
struct TilePages {
    int first, second;
    __device__ inline bool both() const { return first >= 0 && second >= 0; }
};
__device__ inline TilePages tile_pages(const Pages& at, const int* pages, int tile, int end) {
    // the table is read by scalar loads: nothing writes it while the kernel runs, and pages are the same for the whole wave
    typedef const int __attribute__((address_space(4)))* table_t;
    const table_t table = (table_t)(uintptr_t)pages;
    const int n_pages = (int)at.n_pages;
    const int i0 = (int)((unsigned)tile * kTile >> at.shift), i1 = (int)(((unsigned)tile * kTile + 16) >> at.shift);      // places are under 2^31
    TilePages p{tile < end && i0 < at.most ? table[i0] : -1, tile < end && i1 < at.most ? table[i1] : -1};
    if (p.first >= n_pages) p.first = -1;
    if (p.second >= n_pages) p.second = -1;
    return p;
}

// A wave's columns: NQ tiles of 16 with d <= 32 KC components (EXACT: equal), and what they have summed up.
template <class T, int KC, int NQ, bool EXACT>
struct Columns {
    static constexpr int VT = KC * 2;                // tiles of 16 components
    u32x4 q[NQ][KC];
    f32x4 sums[NQ][VT];
    float reference[NQ], total[NQ];
    int row[NQ];                                     // -1: nothing to do in this column
    uint64_t sees[NQ];                               // rows of a tree

    __device__ inline void start(const AttentionIn& in, long long s, int head, int first_col, int count, uint64_t line, int d, int lane) {
        const int share = in.heads / in.at.kv_heads, col = lane & 15, group = lane >> 4;
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const int x = first_col + t * 16 + col;
            row[t] = x < count * share ? x / share : -1;
            sees[t] = __shfl((unsigned long long)line, max(row[t], 0) & 63);
            const T* from = (const T*)in.q + (s * in.at.m + max(row[t], 0)) * in.q_stride + (long long)(head * share + x % share) * d + group * 8;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                q[t][c] = row[t] >= 0 && (EXACT || c * 32 + group * 8 < d) ? *reinterpret_cast<const u32x4*>(from + c * 32) : u32x4{};
                if (in.negative) q[t][c] ^= 0x80008000u;
            }
            reference[t] = -INFINITY;
            total[t] = 0.f;
#pragma unroll
            for (int v = 0; v < VT; ++v) sums[t][v] = f32x4{};
        }
    }

    // S of a tile: the product of its keys, whose rows are dealt as key_place says, and the queries
    __device__ inline void scores(const u32x4 (&keys)[2][KC], f32x4 (&score)[NQ][2]) const {
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 acc{};
#pragma unroll
                for (int c = 0; c < KC; ++c) acc = multiply<T>(keys[h][c], q[t][c], acc);
                score[t][h] = acc;
            }
    }

    // Bits of 8 places, from `first_place` on, that column t sees; there: their page is.
    __device__ inline unsigned seen(const AttentionIn& in, int t, int first_place, int len, bool there) const {
        const int behind = first_place - len;        // row that the first of them is the place of
        const unsigned cached = behind >= 0 ? 0u : (1u << min(-behind, 8)) - 1;
        unsigned rows;
        if (in.parents) rows = behind >= 64 || behind <= -8 ? 0u : (unsigned)(behind >= 0 ? sees[t] >> behind : sees[t] << -behind);
        else rows = (1u << min(max(row[t] - behind + 1, 0), 8)) - 1;
        return there && row[t] >= 0 ? (cached | rows) & 0xFF : 0u;
    }
    // What columns do not see of the lane's places becomes -inf.
    __device__ inline void mask(const AttentionIn& in, f32x4 (&score)[NQ][2], int first_place, int len, bool there) const {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const unsigned bits = seen(in, t, first_place, len, there);
#pragma unroll
            for (int j = 0; j < 8; ++j) score[t][j >> 2][j & 3] = bits >> j & 1 ? score[t][j >> 2][j & 3] : -INFINITY;
        }
    }
    // 0 times infinity is no number, so in a tile that not every column sees whole such values must not meet weights of 0: those of places without a row
    // (bits of `holds` unset, by halves of words) go, and infinities and NaNs of rows become 0.  -> whether there were any.
    __device__ inline bool tame(u32x4 (&values)[VT], const u32x4& holds) const {
        constexpr uint32_t kOnes = std::is_same<T, half_t>::value ? 0x7C00u : 0x7F80u;
        bool odd = false;
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x = values[v][i] & holds[i];
                const bool low = (x & kOnes) == kOnes, high = (x & kOnes << 16) == kOnes << 16;
                x = low ? x & 0xFFFF0000u : x;
                x = high ? x & 0xFFFFu : x;
                odd |= low | high;
                values[v][i] = x;
            }
        return odd;
    }
    // What the infinities and NaNs that tame() took make of the sums: themselves in every column that sees them, or NaN if its weight is 0.
    // Over the tiles [first, end) that are `step` apart; seldom called, so slow and small.
    __device__ inline void add_odd(const AttentionIn& in, long long s, int head, int first_col, int first, int end, int step, int len, int d, int lane) {
        const int col = lane & 15, group = lane >> 4, share = in.heads / in.at.kv_heads;
#pragma unroll 1
        for (int place = first * kTile; place < end * kTile; place = place % kTile == kTile - 1 ? place + 1 + (step - 1) * kTile : place + 1) {
            const int page = in.at.page_of(s, place), off = place & (in.at.page() - 1);
            if (page < 0) continue;
            const long long base = page * in.at.page_values() + ((long long)head << in.at.shift) * d;
            const T* v_at = (const T*)in.v_cache + base + (off >> 3) * 8 * d + (off & 7);
            const T* k_at = (const T*)in.k_cache + base + off * d;
            bool any = false;
#pragma unroll 1
            for (int c = lane; c < d; c += 64) any |= !(fabsf((float)v_at[c * 8]) < INFINITY);
            if (!__any(any)) continue;
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                if (!(seen(in, t, place, len, true) & 1)) continue;
                const T* x = (const T*)in.q + (s * in.at.m + row[t]) * in.q_stride + (long long)(head * share + (first_col + t * 16 + col) % share) * d;
                float score = 0.f;
#pragma unroll 1
                for (int c = 0; c < d; ++c) score = __builtin_fmaf((float)x[c], (float)k_at[c], score);
                const float w = score == (in.negative ? INFINITY : -INFINITY) ? 0.f : 1.f;
#pragma unroll
                for (int v = 0; v < VT; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int c = v * 16 + group * 4 + i;
                        if (!EXACT && c >= d) continue;
                        const float value = (float)v_at[c * 8];
                        sums[t][v][i] += fabsf(value) < INFINITY ? 0.f : w * value;
                    }
            }
        }
    }

    // Scores, still without the scale, to weights, as the second product's operand (the places 8 group + j are the lane's in both), and the
    // second product.  It takes 16 bits, so a weight is off by up to half a step of the cache's type; what it is divided by stays a sum of fp32 weights.  Root mean square of
    // the results' errors beside 64 bits, relative: 2.1 10^-3 of one bf16 token over 2,049 places, where a result that is only rounded at the end has 1.6 10^-3;
    // 2.3 10^-4 for 2.0 10^-4 of fp16 trees.  (A second product of the weights' rests would take that away for half as many matrix instructions again.)
    __device__ inline void weigh_and_add(f32x4 (&score)[NQ][2], float scale, const u32x4 (&values)[VT]) {
        bool ahead = false;
        float most[NQ];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            // NaN if a score is: the column is NaN then, whatever its reference.  (No inline assembly here: results of matrix instructions have to be waited
            // for, which the compiler does for instructions that it knows.)
            float x = score[t][0][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) x = __builtin_elementwise_maximum(x, score[t][j >> 2][j & 3]);
            most[t] = scale * x;
            ahead |= most[t] > reference[t] + kAhead;
        }
        if (__any(ahead)) {
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                most[t] = fmaxf(most[t], __shfl_xor(most[t], 16));
                most[t] = fmaxf(most[t], __shfl_xor(most[t], 32));
                const float now = fmaxf(reference[t], most[t] - kBelow);
                const float shrink = shrink_by(reference[t], now);
                reference[t] = now;
                total[t] *= shrink;
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] *= shrink;
            }
        }
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const float r = reference[t] == -INFINITY ? 0.f : reference[t];      // nothing seen so far
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = exp2_fast(__builtin_fmaf(score[t][j >> 2][j & 3], scale, -r));
            total[t] += tree_sum<8>(w);
            const u32x4 weights = narrow8<T>(w);
#pragma unroll
            for (int v = 0; v < VT; ++v) sums[t][v] = multiply<T>(values[v], weights, sums[t][v]);
        }
    }

    // a column's lanes hold sums of all its places, but each the total of its own 8 of every 32
    __device__ inline void finish() {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            total[t] += __shfl_xor(total[t], 16);
            total[t] += __shfl_xor(total[t], 32);
            if (row[t] < 0) {                        // went along with the others over the tiles without a mask
                total[t] = 0.f;
                reference[t] = -INFINITY;
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] = f32x4{};
            }
        }
    }

    // piece: where the sums of a part of the places go, -1: these are all.
    __device__ inline void write(const AttentionIn& in, long long s, int head, int block, long long piece, int first_col, int d, int lane) const {
        const int share = in.heads / in.at.kv_heads, col = lane & 15, group = lane >> 4;
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const int x = first_col + t * 16 + col;
            if (x >= in.at.m * share) continue;
            const int h = head * share + x % share;
            const long long flat = s * in.at.m + x / share;
            if (piece >= 0) {
                const long long at = piece * in.cols + (x - block * in.cols);
                if (group == 0) in.norms[at] = make_float2(reference[t], total[t]);
#pragma unroll
                for (int v = 0; v < VT; ++v) {
                    const int c = v * 16 + group * 4;
                    if (EXACT || c < d) *reinterpret_cast<f32x4*>(in.sums + at * d + c) = sums[t][v];
                }
            } else {
                const float by = total[t] == 0.f ? 0.f : 1.f / total[t];
                if (in.lse && group == 0) in.lse[flat * in.heads + h] = total[t] == 0.f ? -INFINITY : (reference[t] + __log2f(total[t])) * kLn2;
                T* to = (T*)in.out + flat * in.out_stride + (long long)h * d + group * 4;
#pragma unroll
                for (int v = 0; v < VT; ++v)
                    if (EXACT || v * 16 + group * 4 < d) {
                        typedef T v4 __attribute__((ext_vector_type(4)));
                        v4 y;
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = (T)(sums[t][v][i] * by);
                        *reinterpret_cast<v4*>(to + v * 16) = y;
                    }
            }
        }
    }
};

// What a workgroup does: a block of columns of a head of a sequence, over tiles of its places.
struct Piece {
    long long s;
    int head, block, len, count, first, end;
    long long places;                                // up to the last that one of the columns sees
    int seen_by_all;                                 // tiles whose places every used column sees, if their pages are there
    long long slot;                                  // where its sums go; -1: they are all of the sequence's
    bool nothing;                                    // no such piece
};

__device__ inline int tiles_of(const AttentionIn& in, int block, int len, int count, long long& places) {
    const int share = in.heads / in.at.kv_heads, used = count * share, last_col = min((block + 1) * in.cols, used) - 1;
    places = block * in.cols >= used ? 0 : in.parents ? (long long)len + count : (long long)len + last_col / share + 1;
    return (int)min((places + kTile - 1) / kTile, (((long long)in.at.most << in.at.shift) + kTile - 1) / kTile);
}

// Without parts a piece is a whole sequence.  With them the tiles of all sequences lie behind each other (each has one at least, whose piece writes its rows
// whatever it finds; fewer than 2^31 in all), a part is as many of these as any other but the last, and a piece is what a part has of a sequence:
// part p's of sequence s is number p + s.
__device__ inline Piece piece_of(const AttentionIn& in, int lane) {
    // blocks of columns that read the same places are 8 workgroups apart: on one XCD, whose L2 they share
    const unsigned order = blockIdx.x, turn = order / 8, n = (unsigned)in.n, kv_heads = (unsigned)in.at.kv_heads;      // under 2^23 workgroups
    const unsigned pass = turn / in.blocks * 8 + order % 8;
    Piece p{};
    p.block = (int)(turn % in.blocks);
    p.slot = -1;
    unsigned part = 0, before = 0, each = 0;         // before: tiles of the sequences before this one; each: of a part
    if (!in.parts) {
        p.nothing = pass >= n * kv_heads;
        if (p.nothing) return p;
        p.s = pass % n;
        p.head = (int)(pass / n);
    } else {
        p.nothing = pass >= kv_heads * (unsigned)(in.parts + in.n);
        if (p.nothing) return p;
        const unsigned number = pass / kv_heads;
        p.head = (int)(pass - number * kv_heads);
        const auto tiles = [&](unsigned s) {
            long long places;
            return s < n ? (unsigned)max(tiles_of(in, p.block, in.at.len(s), in.at.count(s), places), 1) : 0u;
        };
        unsigned all = n == 1 ? tiles(0) : 0;
        if (n > 1) {
            for (unsigned s = lane; s < n; s += 64) all += tiles(s);
            for (int off = 32; off; off >>= 1) all += __shfl_xor(all, off);
        }
        all = __builtin_amdgcn_readfirstlane(all);
        each = (all + in.parts - 1) / in.parts;
        if (n == 1) p.nothing = number * each >= all;
        uint64_t found = n == 1;
        for (unsigned base = 0; base < n && !found; base += 64) {
            const unsigned mine = tiles(base + lane);
            unsigned upto = mine;
            for (int off = 1; off < 64; off <<= 1) {
                const unsigned below = __shfl_up(upto, off);
                if (lane >= off) upto += below;
            }
            const unsigned of = number - (base + lane), from = before + upto - mine;      // of: the part, if it has a share of the lane's sequence
            found = __ballot(mine > 0 && number >= base + lane && of < (unsigned)in.parts && max(of * each, from) < min((of + 1) * each, before + upto));
            if (found) {
                const int l = __ffsll((unsigned long long)found) - 1;
                p.s = __builtin_amdgcn_readfirstlane(base + l);
                before = __shfl(from, l);
            } else before += __shfl(upto, 63);
        }
        p.nothing = p.nothing || !found;
        if (p.nothing) return p;
        part = number - (unsigned)p.s;
        before = __builtin_amdgcn_readfirstlane(before);
    }
    p.len = __builtin_amdgcn_readfirstlane(in.at.len(p.s));
    p.count = __builtin_amdgcn_readfirstlane(in.at.count(p.s));
    const int tiles = tiles_of(in, p.block, p.len, p.count, p.places);
    p.end = tiles;
    if (in.parts) {
        const unsigned start = part * each;
        p.first = start > before ? min((int)(start - before), tiles) : 0;
        p.end = (int)min(start + each - before, (unsigned)tiles);
        // the parts that the sequence's first and last tile are in
        const unsigned first = before / each, last = (before + max(tiles, 1) - 1) / each;
        if (first != last) p.slot = ((long long)p.head * in.blocks + p.block) * (in.parts + in.n) + part + p.s;
        if (part == first && p.head == 0 && threadIdx.x == 0) in.spans[p.s * in.blocks + p.block] = make_int2((int)first, (int)last);
    }
    // of a chain's rows those up to the block's first
    p.seen_by_all = min((int)(((long long)p.len + (in.parents ? 0 : p.block * in.cols / (in.heads / in.at.kv_heads) + 1)) / kTile), p.end);
    return p;
}

// The place of a tile whose key the lane `lane` holds in the first half of the first product's rows; 4 more in the second.
__device__ inline int key_place(int lane) { return ((lane & 15) >> 2) * 8 + (lane & 3); }

// The halves of words that hold values of places which are there: of the 8 places from first_place on.
__device__ inline u32x4 held_fields(bool there, int first_place, long long places) {
    u32x4 holds;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        holds[i] = (there && first_place + 2 * i < places ? 0xFFFFu : 0u) | (there && first_place + 2 * i + 1 < places ? 0xFFFF0000u : 0u);
    return holds;
}

// Few columns: the four waves share them, take every fourth tile, and add up at the end.  Keys and values come from the cache into registers, the next
// tile's as soon as this one's are used: every byte of the cache is read once.  Bound by HBM: one row of 32 sequences of up to 16,384 places, 32 heads of 128 over
// 8, 257 us (1.35 GB, 5.3 TB/s of the 5.6 that a plain read reaches).
template <class T, int KC, int NQ, bool EXACT>
__global__ __launch_bounds__(kAttentionThreads) void attention_shared_kernel(AttentionIn in) {
    constexpr int VT = KC * 2, STEP = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, group = lane >> 4;
    const int d = EXACT ? KC * 32 : in.at.d;
    __shared__ float refs[4][NQ][16], totals[4][NQ][16];
    __shared__ f32x4 shared[2][NQ][VT][64];
    const Piece p = piece_of(in, lane);
    if (p.nothing) return;
    const int end = p.end, len = p.len;
    Columns<T, KC, NQ, EXACT> cols;
    cols.start(in, p.s, p.head, p.block * NQ * 16, p.count, in.parents ? tree_line(in, p.s, p.count, lane) : 0, d, lane);

    const int* pages = in.at.pages + p.s * in.at.stride;
    const long long page_values = in.at.page_values();
    const int in_page = in.at.page() - 1;
    const bool second_k = col >> 3, second_v = group >> 1;          // in the tile's second 16 places
    const int k_lane = (key_place(lane) & 15) * d + group * 8, v_lane = (group & 1) * 8 * d + col * 8;
    const T* const k_head = (const T*)in.k_cache + ((long long)p.head << in.at.shift) * d;
    const T* const v_head = (const T*)in.v_cache + ((long long)p.head << in.at.shift) * d;
    u32x4 keys[2][KC], values[VT];
    const auto load_keys = [&](int tile, const TilePages& at) {
        const int off0 = (tile * kTile) & in_page, off1 = (tile * kTile + 16) & in_page;
        const T* from = k_head + (second_k ? max(at.second, 0) * page_values + off1 * d : max(at.first, 0) * page_values + off0 * d) + k_lane;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < KC; ++c) keys[t][c] = EXACT || c * 32 + group * 8 < d ? *reinterpret_cast<const u32x4*>(from + t * 4 * d + c * 32) : u32x4{};
    };
    const auto load_values = [&](int tile, const TilePages& at) {
        const int off0 = (tile * kTile) & in_page, off1 = (tile * kTile + 16) & in_page;
        const T* from = v_head + (second_v ? max(at.second, 0) * page_values + off1 * d : max(at.first, 0) * page_values + off0 * d) + v_lane;
#pragma unroll
        for (int v = 0; v < VT; ++v) values[v] = EXACT || v * 16 + col < d ? *reinterpret_cast<const u32x4*>(from + v * 128) : u32x4{};
    };

    int tile = p.first + wave;
    TilePages now = tile_pages(in.at, pages, tile, end), next = tile_pages(in.at, pages, tile + STEP, end);
    if (tile < end) {
        load_keys(tile, now);
        load_values(tile, now);
    }
    bool odd = false;
    const auto go = [&](auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const TilePages after = tile_pages(in.at, pages, tile + 2 * STEP, end);
        const bool more = tile + STEP < end;
        f32x4 score[NQ][2];
        cols.scores(keys, score);
        if (more) load_keys(tile + STEP, next);
        if constexpr (MASKED) {
            const int first_place = tile * kTile + group * 8;
            const bool there = second_v ? now.second >= 0 : now.first >= 0;
            cols.mask(in, score, first_place, len, there);
            odd |= cols.tame(values, held_fields(there, first_place, p.places));
        }
        cols.weigh_and_add(score, in.scale, values);
        if (more) load_values(tile + STEP, next);
        now = next, next = after;
        tile += STEP;
    };
    // tiles of places that every column sees, then those with rows, or (seldom) all from the first that lacks a page
    while (tile < p.seen_by_all && now.both()) go(std::false_type{});
    const int first_masked = tile;
    while (tile < end) go(std::true_type{});
    if (__any(odd)) cols.add_odd(in, p.s, p.head, p.block * NQ * 16, first_masked, end, STEP, len, d, lane);

    cols.finish();
    // the waves' sums about the largest of their references, added up in a fixed order: 0 + 2, 1 + 3, then both
    if (group == 0)
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            refs[wave][t][col] = cols.reference[t];
            totals[wave][t][col] = cols.total[t];
        }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        float most = -INFINITY, sum = 0.f;
        for (int w = 0; w < 4; ++w) most = fmaxf(most, refs[w][t][col]);
        for (int w = 0; w < 4; ++w) sum += totals[w][t][col] * shrink_by(refs[w][t][col], most);
        const float shrink = shrink_by(cols.reference[t], most);
#pragma unroll
        for (int v = 0; v < VT; ++v) cols.sums[t][v] *= shrink;
        cols.reference[t] = most;
        cols.total[t] = sum;
    }
    for (int half = 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) shared[wave - half][t][v][lane] = cols.sums[t][v];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) cols.sums[t][v] += shared[wave][t][v][lane];
        __syncthreads();
    }
    if (wave == 0) cols.write(in, p.s, p.head, p.block, p.slot, p.block * NQ * 16, d, lane);
}

// Many columns: each wave has its own and goes over all tiles, which pass through the LDS, AT_ONCE between two barriers.  A tile is 4 KC operands of a wave, 1 KB
// each in the order of the lanes, so that they come and go in whole lines: 2 KC of keys, then 2 KC of values.  A wave brings MINE of them: from the
// cache into registers three steps before they are used, into the LDS two steps before; the next tile's keys are read from there while this one's scores
// become weights.
//
// 1,024 rows over 7,001 places, 32 heads of 128 over 8, 137 us (160 after a pause): 920 TFLOP/s of the 1,430 of the library's product of 8,192^3.  With eight waves of 32 columns a tile
// takes a CU 2,900 clocks, 1,024 of them matrix instructions (counters: the vector ALU is busy 1,450, and waves wait for barriers, the LDS and each other).  Four
// waves of 64 columns (half the LDS reads) do not fit the registers: what is scaled now and then has to be where matrix instructions do not keep
// it, and moves cost more.  Two phases a tile, half of the waves one behind: 175 us and no room for the masked tiles.  Left out in copies: exponentials -15 us, half of
// the second product -30, the cache -16.
template <class T, int KC, int NQ, int WAVES, bool EXACT>
__global__ __launch_bounds__(64 * WAVES) void attention_tiles_kernel(AttentionIn in) {
    constexpr int VT = KC * 2, PARTS = 4 * KC, MINE = PARTS / WAVES, AT_ONCE = WAVES == 8 ? 2 : 1;
    __shared__ u32x4 stage[3][AT_ONCE][PARTS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, group = lane >> 4;
    const int d = EXACT ? KC * 32 : in.at.d;
    const Piece p = piece_of(in, lane);
    if (p.nothing) return;
    const int end = p.end, len = p.len;
    const int first_col = (p.block * WAVES + wave) * NQ * 16;
    Columns<T, KC, NQ, EXACT> cols;
    cols.start(in, p.s, p.head, first_col, p.count, in.parents ? tree_line(in, p.s, p.count, lane) : 0, d, lane);

    const int* pages = in.at.pages + p.s * in.at.stride;
    const long long page_values = in.at.page_values();
    const int in_page = in.at.page() - 1;
    const bool for_values = wave >= WAVES / 2;
    const int part = wave * MINE % (2 * KC);         // of the keys' or the values' operands
    const bool second = for_values ? group >> 1 : col >> 3;         // in the tile's second 16 places
    const int from_lane = for_values ? (group & 1) * 8 * d + col * 8 + part * 128 : (key_place(lane) & 15) * d + group * 8 + part / KC * 4 * d + part % KC * 32;
    const T* const from_head = (const T*)(for_values ? in.v_cache : in.k_cache) + ((long long)p.head << in.at.shift) * d + from_lane;
    const int apart = for_values ? 128 : 32;
    struct StepPages {
        TilePages of[AT_ONCE];
        __device__ inline bool all() const {
            bool every = true;
            for (int u = 0; u < AT_ONCE; ++u) every = every && of[u].both();
            return every;
        }
    };
    const auto find = [&](int tile) {
        StepPages to;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) to.of[u] = tile_pages(in.at, pages, tile + u, end);
        return to;
    };
    u32x4 ahead[AT_ONCE][MINE];                      // the wave's operands of a step
    const auto bring = [&](int tile, const StepPages& at) {         // (a tile behind the last is read as page 0)
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int off0 = ((tile + u) * kTile) & in_page, off1 = ((tile + u) * kTile + 16) & in_page;
            const T* from = from_head + (second ? max(at.of[u].second, 0) * page_values + off1 * d : max(at.of[u].first, 0) * page_values + off0 * d);
#pragma unroll
            for (int i = 0; i < MINE; ++i) {         // MINE divides KC: keys of one half
                const bool some = EXACT || (for_values ? (part + i) * 16 + col < d : (part % KC + i) * 32 + group * 8 < d);
                ahead[u][i] = some ? *reinterpret_cast<const u32x4*>(from + i * apart) : u32x4{};
            }
        }
    };
    const auto put = [&](int to) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int i = 0; i < MINE; ++i) stage[to][u][wave * MINE + i][lane] = ahead[u][i];
    };
    u32x4 keys[2][KC], values[VT];
    const auto read_keys = [&](const u32x4 (*from)[64]) {
#pragma unroll
        for (int i = 0; i < 2 * KC; ++i) keys[i / KC][i % KC] = from[i][lane];
    };
    int tile = p.first, at = 0;                      // the stage that this step is in
    StepPages now = find(tile), next = find(tile + AT_ONCE), third = find(tile + 2 * AT_ONCE), fourth = find(tile + 3 * AT_ONCE);
    if (tile < end) {
        bring(tile, now);
        put(0);
        if (tile + AT_ONCE < end) {
            bring(tile + AT_ONCE, next);
            put(1);
        }
        if (tile + 2 * AT_ONCE < end) bring(tile + 2 * AT_ONCE, third);
        __syncthreads();
        read_keys(stage[0][0]);
    }
    bool odd = false;
    const auto go = [&](auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const int at1 = at == 2 ? 0 : at + 1, at2 = at1 == 2 ? 0 : at1 + 1;
        __syncthreads();                             // the next step's tiles are there, and the stage of the one before is free
        if (tile + 2 * AT_ONCE < end) put(at2);
        if (tile + 3 * AT_ONCE < end) bring(tile + 3 * AT_ONCE, fourth);
        const StepPages after = find(tile + 4 * AT_ONCE);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (MASKED && tile + u >= end) break;
            f32x4 score[NQ][2];
#pragma unroll
            for (int i = 0; i < VT; ++i) values[i] = stage[at][u][2 * KC + i][lane];
            cols.scores(keys, score);
            read_keys(u + 1 < AT_ONCE ? stage[at][u + 1 < AT_ONCE ? u + 1 : 0] : stage[at1][0]);      // (behind the last tile: of no meaning)
            if constexpr (MASKED) {
                const int first_place = (tile + u) * kTile + group * 8;
                const bool there = group >> 1 ? now.of[u].second >= 0 : now.of[u].first >= 0;
                cols.mask(in, score, first_place, len, there);
                odd |= cols.tame(values, held_fields(there, first_place, p.places));
            }
            cols.weigh_and_add(score, in.scale, values);
        }
        now = next, next = third, third = fourth, fourth = after;
        tile += AT_ONCE;
        at = at1;
    };
    while (tile + AT_ONCE <= p.seen_by_all && now.all()) go(std::false_type{});
    const int first_masked = tile;
    while (tile < end) go(std::true_type{});
    if (__any(odd)) cols.add_odd(in, p.s, p.head, first_col, first_masked, end, 1, len, d, lane);
    cols.finish();
    cols.write(in, p.s, p.head, p.block, p.slot, first_col, d, lane);
}

// The pieces of a row and head added up, in their order: a thread has 4 components.  Bound by latency where pieces are many and rows few, so eight are loaded at
// once (8 pieces of one row 5.1 us, 5.9 one after the other), by memory where rows are many (64 rows of 16 sequences in two to four pieces 14.3 us, 15.5).
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionIn in, long long threads) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= threads) return;
    const int d = in.at.d, per = d / 4, share = in.heads / in.at.kv_heads;
    const long long at = i / per, row = at / in.heads, s = row / in.at.m;
    const int c = (int)(i - at * per) * 4, h = (int)(at - row * in.heads), head = h / share;
    const int x = (int)(row - s * in.at.m) * share + h % share, block = x / in.cols;
    const int2 span = in.spans[s * in.blocks + block];
    if (span.x == span.y) return;                    // in one piece, and written
    const long long first = ((((long long)head * in.blocks + block) * (in.parts + in.n) + span.x + s) * in.cols) + x % in.cols;
    const int pieces = span.y - span.x + 1;
    float most = -INFINITY;
    // eight pieces' loads at once, the last one's again where there are fewer
    f32x4 sum{};
    float total = 0.f;
    for (int p = 0; p < pieces; p += 8) {
        float2 norm[8];
        f32x4 part[8];
        float now = most;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const long long piece = first + (long long)min(p + j, pieces - 1) * in.cols;
            norm[j] = in.norms[piece];
            part[j] = *reinterpret_cast<const f32x4*>(in.sums + piece * d + c);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) now = fmaxf(now, norm[j].x);
        const float shrink = shrink_by(most, now);
        sum *= shrink;
        total *= shrink;
        most = now;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (p + j >= pieces) break;
            const float by = shrink_by(norm[j].x, most);
            total += norm[j].y * by;
            sum += part[j] * by;
        }
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
    if (in.lse && c == 0) in.lse[at] = total == 0.f ? -INFINITY : (most + __log2f(total)) * kLn2;
    typedef T v4 __attribute__((ext_vector_type(4)));
    v4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (T)(sum[j] * by);
    *reinterpret_cast<v4*>((T*)in.out + row * in.out_stride + (long long)h * d + c) = y;
}

template <class T, int KC, bool EXACT>
int launch_attention(const AttentionIn& in, const AttentionPlan& plan, hipStream_t stream) {
    const long long passes = in.at.kv_heads * (in.parts + in.n);
    const dim3 grid((unsigned)((passes + 7) / 8 * 8 * in.blocks)), threads(64 * plan.waves);
    if (!plan.apart && plan.tiles == 1) hipLaunchKernelGGL((attention_shared_kernel<T, KC, 1, EXACT>), grid, threads, 0, stream, in);
    else if (plan.apart && plan.tiles == 1) hipLaunchKernelGGL((attention_tiles_kernel<T, KC, 1, 4, EXACT>), grid, threads, 0, stream, in);
    else if constexpr (KC <= 4) {
        if (!plan.apart) hipLaunchKernelGGL((attention_shared_kernel<T, KC, 2, EXACT>), grid, threads, 0, stream, in);
        else hipLaunchKernelGGL((attention_tiles_kernel<T, KC, 2, 8, EXACT>), grid, threads, 0, stream, in);
    }
    HIP_TRY(hipGetLastError());
    if (in.parts) {
        const long long all = in.n * in.at.m * in.heads * (in.at.d / 4);       // few, or the places would not be divided
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3((unsigned)((all + 255) / 256)), dim3(256), 0, stream, in, all);
        HIP_TRY(hipGetLastError());
    }
    return IVFPQ_OK;
}

template <class T>
int launch_attention(const AttentionIn& in, const AttentionPlan& plan, hipStream_t stream) {
    switch (in.at.d) {
        case 64: return launch_attention<T, 2, true>(in, plan, stream);
        case 128: return launch_attention<T, 4, true>(in, plan, stream);
        case 256: return launch_attention<T, 8, true>(in, plan, stream);
    }
    if (in.at.d < 64) return launch_attention<T, 2, false>(in, plan, stream);
    if (in.at.d < 128) return launch_attention<T, 4, false>(in, plan, stream);
    return launch_attention<T, 8, false>(in, plan, stream);
}

// Shapes that the call takes; what their launches need fits the launches' limits.
bool known_shape(int64_t n, int32_t m, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_places) {
    return n >= 1 && n <= (1 << 20) && m >= 1 && m <= kMostChain && n * m <= (1 << 24) && kv_heads >= 1 && kv_heads <= 4096 && heads >= kv_heads &&
           heads % kv_heads == 0 && heads <= 65536 && d >= 8 && d <= kMostHead && d % 8 == 0 && max_places >= 0 && max_places < kMostPlaces + kMostChain &&
           n * m * heads <= ((int64_t)1 << 26);
}
// a launch has fewer than 2^32 threads
bool fits_launch(int64_t n, int32_t kv_heads, const AttentionPlan& plan) { return (plan.parts + n) * kv_heads * plan.blocks <= ((int64_t)1 << 23); }

}  // namespace

extern "C" {

size_t ivfpq_draft_attention_workspace_bytes(int64_t n, int32_t m, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_places) {
    if (!known_shape(n, m, heads, kv_heads, d, max_places)) return 0;
    const AttentionPlan plan = attention_plan(n, m, heads, kv_heads, d, max_places);
    return align_up((size_t)attention_scratch_bytes(n, kv_heads, d, plan));
}

int ivfpq_draft_attention(const void* d_q, int64_t q_stride, int32_t heads, int64_t n, int32_t m, const int32_t* d_parents, const int32_t* d_counts,
                          const void* d_k_cache, const void* d_v_cache, int32_t cache_dtype, int64_t n_pages, int32_t kv_heads, int32_t page,
                          int32_t d, const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, int64_t max_places, float scale, void* d_out,
                          int64_t out_stride, float* d_lse, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded("ivfpq_draft_attention", [&] {
        const char* what = "ivfpq_draft_attention";
        if (int rc = check_cache(what, d_k_cache, d_v_cache, cache_dtype, n_pages, kv_heads, page, d, d_pages, max_pages, d_lens, n, m)) return rc;
        if (heads < kv_heads || heads % kv_heads) return fail(IVFPQ_EINVAL, "%s: heads=%d is no multiple of kv_heads=%d", what, heads, kv_heads);
        if (d_parents && m > IVFPQ_MAX_DRAFT) return fail(IVFPQ_EUNSUPPORTED, "%s: a tree of m=%d rows (limit %d)", what, m, (int)IVFPQ_MAX_DRAFT);
        if (max_places < 0) return fail(IVFPQ_EINVAL, "%s: max_places=%lld", what, (long long)max_places);
        if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return fail(IVFPQ_EINVAL, "%s: the scale is not finite", what);
        if (n == 0) return (int)IVFPQ_OK;
        if (!known_shape(n, m, heads, kv_heads, d, max_places)) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld m=%d heads=%d max_places=%lld: over the limits (2^26 rows and heads)", what, (long long)n, m, heads, (long long)max_places);
        if (!d_q || !d_out) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        const int64_t rows = n * m;
        if (rows > 1 && (q_stride < (int64_t)heads * d || out_stride < (int64_t)heads * d || q_stride % 8 || out_stride % 4))
            return fail(IVFPQ_EINVAL, "%s: a row stride below the row's values, or no multiple of 8 (queries) or 4 (output)", what);
        if ((uintptr_t)d_q % 16 || (uintptr_t)d_out % 8 || (uintptr_t)d_lse % 4) return fail(IVFPQ_EINVAL, "%s: queries are not aligned to 16 bytes, or the output not to 8", what);
        AttentionPlan plan = attention_plan(n, m, heads, kv_heads, d, max_places);
        if (!tiles_numbered(n, (int64_t)max_pages * page)) plan.parts = 0;
        if (!fits_launch(n, kv_heads, plan)) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld m=%d heads=%d kv_heads=%d: over 2^23 workgroups", what, (long long)n, m, heads, kv_heads);
        const size_t need = align_up((size_t)attention_scratch_bytes(n, kv_heads, d, plan));
        if (need) {
            if (!d_workspace) return fail(IVFPQ_EINVAL, "%s: null workspace", what);
            if ((uintptr_t)d_workspace % kAlign) return fail(IVFPQ_EINVAL, "%s: workspace not aligned to %zu bytes", what, kAlign);
            if (workspace_bytes < need) return fail(IVFPQ_ENOSPACE, "%s: workspace %zu bytes, need %zu", what, workspace_bytes, need);
        }
        AttentionIn in{d_q, d_k_cache, d_v_cache, d_out, d_lse, (float*)d_workspace, nullptr, nullptr, d_parents, q_stride, out_stride, n, heads, plan.blocks, plan.parts, plan.columns(),
                       (float)std::min(std::max(std::abs((double)scale) * 1.4426950408889634, 1e-37), 3e38), scale < 0.f, pages_in(d_pages, max_pages, d_lens, d_counts, n_pages, kv_heads, page, d, m)};
        const size_t pieces = (size_t)attention_pieces(n, kv_heads, plan);
        in.norms = (float2*)(in.sums + pieces * d);        // d is a multiple of 8
        in.spans = (int2*)(in.norms + pieces);
        // what is looked at ends with the table, wherever max_places is: lengths may have grown since a call was captured
        if (!n_pages) in.at.most = 0;
        return with_value_type(cache_dtype, [&](auto t) {
            using T = decltype(t);
            if constexpr (sizeof(T) == 4) return (int)IVFPQ_EINVAL;
            else return launch_attention<T>(in, plan, (hipStream_t)hip_stream);
        });
    });
}

}  // extern "C"
