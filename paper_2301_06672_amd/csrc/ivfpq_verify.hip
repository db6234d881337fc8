// Drafted tokens against the model's logits: what ivfpq_verify_drafts does.
//
// A token is drawn by where a given number falls among sums of probabilities, and as many borders as there are tokens lie close together, so sums are of
// 64 bits and their terms right to 1.1 10^-12.  A row is read once, in blocks whose largest logit and sum about it are kept; where a token is drawn, the
// sums say in which block, and that block is read again.  Two exponentials, both with polynomials interpolated at Chebyshev's points: the terms of the blocks' sums are
// 2^n 2^(i / 32) 2^(f / 32) with a table of 32 powers and degree 4 (off by 8 10^-14 at most), as there are many; everything else (what scales a
// block's sum, the tokens of a block that is read again, a student's remainder) is 2^n 2^f with degree 8 (off by 1.1 10^-12).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_values.hpp"

using namespace ivfpq;

namespace {

constexpr int kMostDraft = IVFPQ_MAX_DRAFT;
constexpr int kBlock = 2048;                          // values of a block, one wave's work: 32 a lane
constexpr int kLaneValues = kBlock / 64;
constexpr int kLeftBlock = 512;                       // of what a draft leaves of a distribution: few rows, so more waves for each
constexpr int kLeftValues = kLeftBlock / 64;

// What is kept of a block: the sum of exp((x - most) / T).  NaN and +inf stay in `most`.
struct BlockSum {
    double sum;
    float most;
    int unused;
};

// What a row says: its token (-1: none) and the logarithm of its probability.
struct Said {
    int token;
    float chance;
};

struct VerifyIn {
    const void *logits, *drafts;
    long long stride, draft_stride;
    const int *tokens, *parents, *counts;             // [n][m]; parents, counts or null
    const float *uniforms, *accept;                   // [n][m] or null
    BlockSum* blocks;                                 // [n * m + n * (m - 1) with drafts][row_blocks]
    double* left;                                     // drafts: [n][left_blocks]
    struct Stop* stops;                               // drafts: [n]
    Said* said;                                       // without drafts: [n * m]
    int *path, *kept, *next;
    float* logprobs;
    long long n;
    int m, vocab, row_blocks, left_blocks;
    double scale;                                     // log2(e) / T
    __device__ inline int count(long long s) const { return counts ? min(max(counts[s], 0), m) : m; }
};

// Where a sequence's chain ends: the row whose distribution the next token comes from, and what normalises it and its draft's.
struct Stop {
    float most, draft_most;
    double total;                                     // 0: no distribution
    double of_total, of_draft;                        // 1 by it and by the draft's
    int row, drafted;                                 // row -1: no used rows; drafted: less the draft's probabilities
};

__device__ inline float maximum3(float a, float b, float c) {       // NaN if one of them is
    float d;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// 2^y for y <= 1/2, right to 1.1 10^-12; what is under 2^-1000 may be anything down to 0
__device__ inline double exp2_exact(double y) {
    y = fmax(y, -1100.0);
    const double n = rint(y), f = y - n;
    double p = 0x1.63d1363a7ecb6p-20;
    p = fma(p, f, 0x1.00dc4a534054dp-16);
    p = fma(p, f, 0x1.4308ac85a6c21p-13);
    p = fma(p, f, 0x1.5d8745a72827ap-10);
    p = fma(p, f, 0x1.3b2ab7181b778p-7);
    p = fma(p, f, 0x1.c6b08dd6fd236p-5);
    p = fma(p, f, 0x1.ebfbdff823cedp-3);
    p = fma(p, f, 0x1.62e42fef84cf0p-1);
    p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}
// 2^(i / 32)
__device__ const double kExp2Table[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0, 0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0,
    0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0, 0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0, 0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0,
    0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0, 0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0, 0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0,
    0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};
// 2^(y / 32) in fewer instructions, right to 8 10^-14, from the nearest whole number of y and the rest: 2^(n + i / 32 + f / 32) with 2^(i / 32) from a table in
// the LDS, n added to its exponent, and a polynomial of degree 4 for the rest, |f| <= 1/2.  An addition leaves the nearest whole number in the low bits.
// The coefficients stay in vector registers: an operation takes one from a scalar register at most, and a copy of it costs as much as the operation.
constexpr int kExp2Steps = 32;
constexpr double kWhole = 0x1.8p52;
__device__ inline int low_word(double x) { return __builtin_bit_cast(int2, x).x; }
struct Exp2Terms {
    const double* steps;                              // 2^(i / 32) less i 2^15 in the high word, which n 2^20 + i 2^15 is added to
    double c[5] = {1.0, 0x1.62e42fef6d01ap-6, 0x1.ebfbdff8131c3p-13, 0x1.c6b167e571135p-20, 0x1.3b2b1bee88b09p-27};
    __device__ inline Exp2Terms(const double* steps) : steps(steps) {
#pragma unroll
        for (int i = 0; i < 5; ++i) asm("" : "+v"(c[i]));
    }
    // sum + 2^((whole + f) / 32), -32700 < whole < 32700
    __device__ inline double add(int whole, double f, double sum) const {
        int2 step = __builtin_bit_cast(int2, steps[whole & (kExp2Steps - 1)]);
        asm("" : "+v"(step.y));                       // or else the sum is made of 64 bits, in five instructions
        step.y = (int)(((unsigned)whole << 15) + (unsigned)step.y);
        double p = c[4];
#pragma unroll
        for (int i = 3; i >= 0; --i) p = fma(p, f, c[i]);
        return fma(p, __builtin_bit_cast(double, step), sum);
    }
};
// exp((x - most) / T); `most` is finite
__device__ inline double weight(float x, float most, double scale) { return exp2_exact(((double)x - (double)most) * scale); }

// x of another lane by the data paths between lanes, `none` where that lane does not exist (a step of a scan)
template <int CTRL, int ROWS>
__device__ inline int other_lane(int none, int x) { return __builtin_amdgcn_update_dpp(none, x, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ inline double plus_other_lane(double x) {
    const int2 bits = __builtin_bit_cast(int2, x);
    return x + __builtin_bit_cast(double, make_int2(other_lane<CTRL, ROWS>(0, bits.x), other_lane<CTRL, ROWS>(0, bits.y)));
}
// the sum over the lanes up to this one: within rows of 16 lanes by shifts of 1, 2, 4 and 8, then the last lanes of rows spread to the rows behind
__device__ inline double wave_scan(double x) {
    x = plus_other_lane<0x111, 0xF>(x);
    x = plus_other_lane<0x112, 0xF>(x);
    x = plus_other_lane<0x114, 0xF>(x);
    x = plus_other_lane<0x118, 0xF>(x);
    x = plus_other_lane<0x142, 0xA>(x);
    return plus_other_lane<0x143, 0xC>(x);
}
__device__ inline double from_lane(double x, int lane) {
    const int2 bits = __builtin_bit_cast(int2, x);
    return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_readlane(bits.x, lane), __builtin_amdgcn_readlane(bits.y, lane)));
}
__device__ inline double wave_sum(double x) { return from_lane(wave_scan(x), 63); }
template <int CTRL, int ROWS>
__device__ inline float most_of_lanes(float x) {
    const float other = __int_as_float(other_lane<CTRL, ROWS>(__float_as_int(x), __float_as_int(x)));
    return maximum3(x, other, other);
}
// NaN if one is
__device__ inline float wave_maximum(float x) {
    x = most_of_lanes<0x111, 0xF>(x);
    x = most_of_lanes<0x112, 0xF>(x);
    x = most_of_lanes<0x114, 0xF>(x);
    x = most_of_lanes<0x118, 0xF>(x);
    x = most_of_lanes<0x142, 0xA>(x);
    x = most_of_lanes<0x143, 0xC>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ inline bool bad_most(float most) { return !(most < INFINITY); }       // NaN or +inf in the row

// A block of a row as the wave's chunks: chunk i * 64 + lane holds VEC consecutive values, -inf outside of the row.
template <class T>
struct BlockChunks {
    static constexpr int N = kLaneValues / Chunk<T>::VEC;
    Chunk<T> chunk[N];
    __device__ BlockChunks(const RowChunks<T>& row, int block, int lane) {
        const int first = block * (kBlock / Chunk<T>::VEC);
        if (first >= row.first_whole() && first + N * 64 <= row.end_whole()) {
#pragma unroll
            for (int i = 0; i < N; ++i) chunk[i].bits = row.base[first + i * 64 + lane];
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = first + i * 64 + lane;
                if (c < row.count()) chunk[i] = row.load(c);
                else {
                    float none[Chunk<T>::VEC];
#pragma unroll
                    for (int e = 0; e < Chunk<T>::VEC; ++e) none[e] = -INFINITY;
                    chunk[i].narrow(none);
                }
            }
        }
    }
};

// The largest and the smallest of a lane's values.  (Where the smallest is not too far down, no term of the sum has to be looked at for that.)  16-bit ones are compared two at a time as whole numbers: as signed ones the largest is right if it is not
// negative, as unsigned ones the smallest is the largest if all have a sign, and the largest the smallest if one has.
template <class T>
struct Extent {
    float most, least;                                // most: NaN if a value is
    __device__ inline Extent(const BlockChunks<T>& held) {
        if constexpr (sizeof(T) == 2) {
            typedef int16_t s2 __attribute__((ext_vector_type(2)));
            typedef uint16_t u2 __attribute__((ext_vector_type(2)));
            constexpr unsigned kInf = std::is_same<T, half_t>::value ? 0x7C00 : 0x7F80;
            s2 top = __builtin_bit_cast(s2, held.chunk[0].bits.x);
            u2 high = __builtin_bit_cast(u2, top), low = high;
#pragma unroll
            for (int i = 0; i < held.N; ++i) {
                const uint4 bits = held.chunk[i].bits;
                const uint32_t words[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(s2, words[j]));
                    high = __builtin_elementwise_max(high, __builtin_bit_cast(u2, words[j]));
                    low = __builtin_elementwise_min(low, __builtin_bit_cast(u2, words[j]));
                }
            }
            const int largest = max(top.x, top.y);
            const unsigned highest = max(high.x, high.y), lowest = min(low.x, low.y);
            const auto value = [](unsigned bits) { return (float)__builtin_bit_cast(T, (uint16_t)bits); };
            most = highest > (0x8000 | kInf) ? NAN : value(largest >= 0 ? (unsigned)largest : lowest);
            least = value(highest >= 0x8000 ? highest : lowest);
        } else {
            most = -INFINITY, least = INFINITY;
#pragma unroll
            for (int i = 0; i < held.N; ++i) {
                float x[4];
                held.chunk[i].widen(x);
                most = maximum3(maximum3(most, x[0], x[1]), x[2], x[3]);
                least = fminf(fminf(least, fminf(x[0], x[1])), fminf(x[2], x[3]));
            }
        }
    }
};

constexpr int kSumThreads = 256;

// The blocks' sums of all used rows, a wave a block.  Bound by vector instructions, 4 clocks of a SIMD each whether of 32 bits or of 64 (counters: busy all the time with
// 730 a wave): 1.5 a value to the extremes, 14 to the sum.  1,024 rows of 65,536 bf16 logits, 134 MB, take 42 us, 24 to read; with a polynomial of degree 8
// in place of the table and every value held above a bound 51.  A table for each wave, filled while the logits are on their way: 45.
template <class T>
__global__ __launch_bounds__(kSumThreads, sizeof(T) == 2 ? 8 : 5) void block_sums_kernel(VerifyIn in) {
    constexpr int VEC = Chunk<T>::VEC;
    __shared__ double steps[kExp2Steps];
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < kExp2Steps) {
        int2 step = __builtin_bit_cast(int2, kExp2Table[threadIdx.x]);
        step.y -= (int)threadIdx.x << 15;
        steps[threadIdx.x] = __builtin_bit_cast(double, step);
    }
    __syncthreads();
    // 2^25 blocks of 2^21 rows at most; divisions of 64 bits would take as long as a third of the sums
    const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kSumThreads / 64) + (threadIdx.x >> 6));
    const unsigned row = item / (unsigned)in.row_blocks, targets = (unsigned)(in.n * in.m);
    const int block = (int)(item - row * in.row_blocks);
    const bool draft = row >= targets;
    const unsigned r = draft ? row - targets : row, per = draft ? in.m - 1 : in.m;
    if (draft && (!in.drafts || r >= (unsigned)in.n * per)) return;
    const unsigned s = r / per;
    // a draft row is used if the row that it drafted is
    if ((int)(r - s * per) + (draft ? 1 : 0) >= in.count(s)) return;
    const RowChunks<T> values(draft ? in.drafts : in.logits, r, draft ? in.draft_stride : in.stride, in.vocab);
    if (block * kBlock >= values.end) return;
    BlockChunks<T> held(values, block, lane);
    const Extent<T> extent(held);
#pragma unroll
    for (int i = 0; i < held.N; ++i) held.chunk[i].forget_widened();
    const float most = wave_maximum(extent.most);
    double sum = 0.0;
    if (most > -INFINITY && most < INFINITY) {
        const Exp2Terms power(steps);
        const double scale = in.scale * kExp2Steps;
        const auto add_up = [&](auto&& add) {
            double sums[2] = {0.0, 0.0};
#pragma unroll
            for (int i = 0; i < held.N; ++i) {
                float x[VEC];
                held.chunk[i].widen(x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sums[e & 1] = add((double)x[e], sums[e & 1]);
            }
            return wave_sum(sums[0] + sums[1]);
        };
        const double whole_most = rint((double)most * scale);
        if (fabs(whole_most) < 0x1p30 && __all(((double)extent.least - (double)most) * scale > -32000.0)) {
            // x scale = r + f; r less that of the largest is in the low bits, and what the largest had of f is a factor of the whole block
            const double magic = kWhole - whole_most;
            sum = add_up([&](double x, double sum) {
                const double shifted = fma(x, scale, magic);
                return power.add(low_word(shifted), fma(x, scale, magic - shifted), sum);
            });
            sum *= exp2_exact(fma((double)most, scale, -whole_most) * (-1.0 / kExp2Steps));
        } else {
            // what is under 2^-1000, of a logit of -inf too, is taken for that: lost in a sum that holds a 1
            sum = add_up([&](double x, double sum) {
                const double y = fmax((x - (double)most) * scale, -32000.0), shifted = y + kWhole;
                return power.add(low_word(shifted), y - (shifted - kWhole), sum);
            });
        }
    }
    if (lane == 0) in.blocks[item] = BlockSum{sum, most, 0};
}

// A row's largest logit and the sum about it, from its blocks; the same in every lane.
struct Norm {
    float most;
    double total;                                     // 0: all -inf; NaN: bad
};
__device__ inline double block_weight(const BlockSum& b, float most, double scale) { return b.most > -INFINITY ? b.sum * weight(b.most, most, scale) : 0.0; }

__device__ inline Norm row_norm(const BlockSum* blocks, int count, double scale, int lane) {
    BlockSum mine{0.0, -INFINITY, 0};                 // of the first 64; a larger vocabulary's others are read twice
    if (lane < count) mine = blocks[lane];
    float most = mine.most;
    for (int b = lane + 64; b < count; b += 64) most = maximum3(most, blocks[b].most, blocks[b].most);
    most = wave_maximum(most);
    if (bad_most(most)) return Norm{most, NAN};
    if (most == -INFINITY) return Norm{most, 0.0};
    double total = block_weight(mine, most, scale);
    for (int b = lane + 64; b < count; b += 64) total += block_weight(blocks[b], most, scale);
    return Norm{most, wave_sum(total)};
}

__device__ inline double unit(float u) {              // into [0, 1)
    return (double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f);
}

// Running sums over the lanes: the first lane at which one that adds something is over `target`, or else the last that adds something; -1 if none does.
// before: the running sum before that lane.  base: the sum before the lanes, and after the call behind them.
struct Crossing {
    int lane;
    bool over;
    double before;
};
__device__ inline Crossing cross(double mine, double target, double& base) {
    const double upto = base + wave_scan(mine);
    const uint64_t some = __ballot(mine > 0.0), over = __ballot(mine > 0.0 && upto > target);
    Crossing c{over ? __ffsll((unsigned long long)over) - 1 : some ? 63 - __clzll((long long)some) : -1, over != 0, base};
    if (c.lane > 0) c.before = from_lane(upto, __builtin_amdgcn_readfirstlane(c.lane) - 1);
    base = from_lane(upto, 63);
    return c;
}

// The first block of `count` whose running sum, `of` it, is over `share` times the sum of all.  -1 if all are 0.
struct Picked {
    int block;
    double before, target;
};
template <class Of>
__device__ inline Picked pick_block(int count, double share, int lane, Of&& of) {
    const double mine = lane < count ? of(lane) : 0.0;
    double all = mine;
    for (int b = lane + 64; b < count; b += 64) all += of(b);
    all = wave_sum(all);
    Picked picked{-1, 0.0, share * all};
    double base = 0.0;
    for (int first = 0; first < count && all > 0.0; first += 64) {
        const Crossing c = cross(first == 0 ? mine : first + lane < count ? of(first + lane) : 0.0, picked.target, base);
        if (c.lane >= 0) {
            picked.block = first + c.lane;
            picked.before = c.before;
        }
        if (c.over) break;
    }
    return picked;
}

// The lowest of a block's tokens whose running sum, with what is before the block, is over the target; -1 if all weigh nothing.  A lane has
// N tokens in a row: their weights w, that lie from token `first` of the row on.
template <int N>
__device__ inline int pick_token(const double (&w)[N], int first, const Picked& picked) {
    double mine = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += w[i];
    double base = picked.before;
    const Crossing c = cross(mine, picked.target, base);
    if (c.lane < 0) return -1;
    double at = c.before;
    int token = -1;
    bool over = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        at += w[i];
        if (w[i] > 0.0 && !over) {
            token = first + i;                        // the last one, where rounding leaves all under the target
            over = at > picked.target;
        }
    }
    return __builtin_amdgcn_readlane(token, __builtin_amdgcn_readfirstlane(c.lane));
}

// The token that a row's distribution has at the share u of its sum, or its most likely one; -1 without a distribution.
template <class T>
__device__ inline int draw(const VerifyIn& in, long long flat, const Norm& norm, bool greedy, double u, int lane, float& logit) {
    if (!(norm.total > 0.0)) return -1;
    constexpr int VEC = Chunk<T>::VEC;
    const RowChunks<T> row(in.logits, flat, in.stride, in.vocab);
    const BlockSum* blocks = in.blocks + flat * in.row_blocks;
    const int count = (row.end + kBlock - 1) / kBlock;
    if (greedy) {
        int block = 0x7FFFFFFF;
        for (int b = lane; b < count; b += 64)
            if (blocks[b].most == norm.most) block = min(block, b);
        for (int off = 32; off; off >>= 1) block = min(block, __shfl_xor(block, off));
        BlockChunks<T> held(row, block, lane);
        int token = 0x7FFFFFFF;
#pragma unroll
        for (int i = 0; i < held.N; ++i) {
            float x[VEC];
            held.chunk[i].widen(x);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (x[e] == norm.most) token = min(token, (block * (kBlock / VEC) + i * 64 + lane) * VEC + e - row.lead);
        }
        for (int off = 32; off; off >>= 1) token = min(token, __shfl_xor(token, off));
        logit = norm.most;
        return token;
    }
    const Picked picked = pick_block(count, u, lane, [&](int b) { return block_weight(blocks[b], norm.most, in.scale); });
    if (picked.block < 0) return -1;
    const float most = blocks[picked.block].most;
    const double by = weight(most, norm.most, in.scale);
    const int first = picked.block * (kBlock / VEC) + lane * (kLaneValues / VEC);       // the lane's chunks lie in a row
    double w[kLaneValues];
#pragma unroll
    for (int i = 0; i < kLaneValues / VEC; ++i) {
        float x[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = -INFINITY;
        if (first + i < row.count()) row.load(first + i).widen(x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[i * VEC + e] = by * weight(x[e], most, in.scale);
    }
    const int token = pick_token(w, first * VEC - row.lead, picked);
    if (token >= 0) logit = row.value(token);
    return token;
}

__device__ inline float log_probability(float logit, const Norm& norm, double scale) {
    return (float)(((double)logit - (double)norm.most) * scale * 0.6931471805599453 - log(norm.total));
}
// of a row from which no token comes
__device__ inline float no_probability(const Norm& norm) { return norm.total == 0.0 ? -INFINITY : NAN; }

template <class T>
__device__ inline int row_block_count(const VerifyIn& in, const void* data, long long r, long long stride) {
    return (RowChunks<T>(data, r, stride, in.vocab).end + kBlock - 1) / kBlock;
}

// The tokens of all used rows, a wave a row: what the sums of its blocks say, then one block again, 32 tokens in a row a lane.  1,024 rows 9 us (43 as 16 waves of one
// workgroup a sequence, with sums between lanes through the LDS): a chain of three reads.
template <class T>
__global__ __launch_bounds__(64) void draw_rows_kernel(VerifyIn in) {
    const int lane = threadIdx.x;
    const long long flat = blockIdx.x, s = flat / in.m;
    if ((int)(flat - s * in.m) >= in.count(s)) return;
    const Norm norm = row_norm(in.blocks + flat * in.row_blocks, row_block_count<T>(in, in.logits, flat, in.stride), in.scale, lane);
    float logit = 0.f;
    const int token = draw<T>(in, flat, norm, !in.uniforms, in.uniforms ? unit(in.uniforms[flat]) : 0.0, lane, logit);
    if (lane == 0) in.said[flat] = Said{token, token < 0 ? no_probability(norm) : log_probability(logit, norm, in.scale)};
}

// The way through a tree, a wave a sequence and a lane a row.
__global__ __launch_bounds__(64) void verify_tree_kernel(VerifyIn in) {
    const int lane = threadIdx.x, m = in.m;
    const long long s = blockIdx.x;
    const int count = in.count(s);
    int up = -1, token = -1;
    Said said{-1, -INFINITY};
    if (lane < count) {
        up = in.parents ? in.parents[s * m + lane] : lane - 1;
        if (up >= lane) up = -1;
        token = in.tokens[s * m + lane];
        said = in.said[s * m + lane];
    }
    int kept = 0, at = 0, following = -1;
    int my_row = -1;                                  // of the path, at place `lane`
    while (kept < count) {                            // a child comes behind its parent
        if (lane == kept) my_row = at;
        ++kept;
        following = __shfl(said.token, at);
        const uint64_t children = __ballot(lane > 0 && lane < count && up == at && token == following && following >= 0);
        if (!children) break;
        at = __ffsll((unsigned long long)children) - 1;
    }
    const float chance = __shfl(said.chance, max(my_row, 0));
    if (lane < m) {
        in.path[s * m + lane] = my_row;
        in.logprobs[s * m + lane] = my_row >= 0 ? chance : -INFINITY;
    }
    if (lane == 0) {
        in.kept[s] = kept;
        in.next[s] = following;
    }
}

constexpr int kWalkThreads = 1024;

// A student's chain: which rows are kept, and the row where it ends.  A workgroup a sequence, a wave a row.
template <class T>
__global__ __launch_bounds__(kWalkThreads) void verify_chain_kernel(VerifyIn in) {
    __shared__ Norm norms[kMostDraft], draft_norms[kMostDraft];
    __shared__ int passes[kMostDraft];                // whether the row behind this one is kept
    __shared__ float chances[kMostDraft];             // log p of the drafted token
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = in.m;
    const long long s = blockIdx.x;
    const int count = in.count(s);
    for (int i = wave; i < count; i += kWalkThreads / 64) {
        const long long flat = s * m + i;
        const Norm norm = row_norm(in.blocks + flat * in.row_blocks, row_block_count<T>(in, in.logits, flat, in.stride), in.scale, lane);
        Norm draft{-INFINITY, 0.0};
        bool pass = false;
        float chance = -INFINITY;
        if (i + 1 < count) {
            const long long r = s * (m - 1) + i;
            draft = row_norm(in.blocks + (in.n * m + r) * in.row_blocks, row_block_count<T>(in, in.drafts, r, in.draft_stride), in.scale, lane);
            if (!(draft.total > 0.0)) draft.total = 0.0;
            const int token = in.tokens[flat + 1];
            if (norm.total > 0.0 && token >= 0 && token < in.vocab) {
                const float x = (float)((const T*)in.logits)[flat * in.stride + token];
                const double p = weight(x, norm.most, in.scale) / norm.total;
                double q = 0.0;
                if (draft.total > 0.0) q = weight((float)((const T*)in.drafts)[r * in.draft_stride + token], draft.most, in.scale) / draft.total;
                pass = unit(in.accept[flat + 1]) * q < p;
                chance = log_probability(x, norm, in.scale);
            }
        }
        if (lane == 0) {
            norms[i] = norm;
            draft_norms[i] = draft;
            passes[i] = pass;
            chances[i] = chance;
        }
    }
    __syncthreads();
    if (wave != 0) return;
    const uint64_t stops = __ballot(lane >= count || !passes[min(lane, max(count - 1, 0))]);
    const int stop = count ? min(__ffsll((unsigned long long)stops) - 1, count - 1) : -1;
    if (lane < m) {
        in.path[s * m + lane] = lane <= stop ? lane : -1;
        if (lane != stop) in.logprobs[s * m + lane] = lane < stop ? chances[lane] : -INFINITY;
    }
    if (lane == 0) {
        in.kept[s] = stop + 1;
        Stop to{};
        to.row = stop;
        if (stop >= 0) {
            to.most = norms[stop].most;
            to.total = norms[stop].total;
            to.drafted = stop + 1 < count && draft_norms[stop].total > 0.0;
            to.draft_most = draft_norms[stop].most;
            to.of_total = 1.0 / norms[stop].total;
            to.of_draft = 1.0 / draft_norms[stop].total;
        }
        in.stops[s] = to;
    }
}

// max(p - q, 0) of kLeftValues tokens, STEP apart, of the row where a chain ends; 0 behind the vocabulary
template <int STEP, class T>
__device__ inline void left_weights(const Stop& stop, const T* logits, const T* drafts, int first, const VerifyIn& in, double (&w)[kLeftValues]) {
    T x[kLeftValues], y[kLeftValues];
#pragma unroll
    for (int i = 0; i < kLeftValues; ++i) {
        const int token = min(first + i * STEP, in.vocab - 1);
        x[i] = logits[token];
        y[i] = drafts[token];
    }
#pragma unroll
    for (int i = 0; i < kLeftValues; ++i) {
        const double p = weight((float)x[i], stop.most, in.scale) * stop.of_total, q = weight((float)y[i], stop.draft_most, in.scale) * stop.of_draft;
        w[i] = first + i * STEP < in.vocab ? fmax(p - q, 0.0) : 0.0;
    }
}
template <class T>
__device__ inline const T* draft_row(const VerifyIn& in, long long s, int i) {
    return (const T*)in.drafts + (s * (in.m - 1) + i) * in.draft_stride;
}

// The sums of max(p - q, 0) over blocks of the rows where chains end, a wave a block: 33 rows of 131,071 in 9.6 us (10 with blocks of 2048, whose 32 tokens a lane then
// take the draw 6.7 us in place of 5.6; 19 with a lane's tokens in a row).  Half of that are its vector instructions, 36 a token.
template <class T>
__global__ __launch_bounds__(kSumThreads) void left_sums_kernel(VerifyIn in) {
    const int lane = threadIdx.x & 63;
    // fewer than 2^26; a division of 64 bits and those of the totals would take longer than the block
    const unsigned item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kSumThreads / 64) + (threadIdx.x >> 6));
    const long long s = item / (unsigned)in.left_blocks;
    const int block = (int)(item - (unsigned)s * in.left_blocks);
    if (s >= in.n) return;
    const Stop stop = in.stops[s];
    if (stop.row < 0 || !stop.drafted || !(stop.total > 0.0)) return;
    const T* x = (const T*)in.logits + (s * in.m + stop.row) * in.stride;
    const T* y = draft_row<T>(in, s, stop.row);
    double w[kLeftValues], sum = 0.0;
    left_weights<64>(stop, x, y, block * kLeftBlock + lane, in, w);
#pragma unroll
    for (int i = 0; i < kLeftValues; ++i) sum += w[i];
    sum = wave_sum(sum);
    if (lane == 0) in.left[s * in.left_blocks + block] = sum;
}

// The next token of a chain, a wave a sequence.
template <class T>
__global__ __launch_bounds__(64) void draw_left_kernel(VerifyIn in) {
    const int lane = threadIdx.x;
    const long long s = blockIdx.x;
    const Stop stop = in.stops[s];
    if (stop.row < 0) {
        if (lane == 0) in.next[s] = -1;
        return;
    }
    const long long flat = s * in.m + stop.row;
    const Norm norm{stop.most, stop.total};
    const double u = unit(in.uniforms[flat]);
    int token = -1;
    float logit = 0.f;
    if (stop.drafted && norm.total > 0.0) {
        const double* left = in.left + s * in.left_blocks;
        const Picked picked = pick_block(in.left_blocks, u, lane, [&](int b) { return left[b]; });
        if (picked.block >= 0) {
            const T* x = (const T*)in.logits + flat * in.stride;
            double w[kLeftValues];
            left_weights<1>(stop, x, draft_row<T>(in, s, stop.row), picked.block * kLeftBlock + lane * kLeftValues, in, w);
            token = pick_token(w, picked.block * kLeftBlock + lane * kLeftValues, picked);
            if (token >= 0) logit = (float)x[token];
        }
    }
    if (token < 0) token = draw<T>(in, flat, norm, false, u, lane, logit);
    if (lane == 0) {
        in.next[s] = token;
        in.logprobs[flat] = token < 0 ? no_probability(norm) : log_probability(logit, norm, in.scale);
    }
}

// ---- launches

int row_blocks(int32_t vocab) { return (int)(((int64_t)vocab + 7 + kBlock - 1) / kBlock); }      // at the worst alignment
int left_blocks(int32_t vocab) { return (int)(((int64_t)vocab + kLeftBlock - 1) / kLeftBlock); }

struct VerifySpace {
    size_t blocks, left, stops, said;
    size_t bytes() const { return blocks + left + stops + said; }
};
VerifySpace verify_space(int64_t n, int32_t m, int32_t vocab, bool drafts) {
    VerifySpace v{};
    v.blocks = align_up((size_t)(n * m + (drafts ? n * (m - 1) : 0)) * row_blocks(vocab) * sizeof(BlockSum));
    if (drafts) {
        v.left = align_up((size_t)n * left_blocks(vocab) * sizeof(double));
        v.stops = align_up((size_t)n * sizeof(Stop));
    } else {
        v.said = align_up((size_t)(n * m) * sizeof(Said));
    }
    return v;
}

constexpr int64_t kMostRows = 1 << 21;
constexpr int64_t kMostBlocks = (int64_t)1 << 25;            // a wave each: a launch has fewer than 2^32 threads

bool verify_shape(int64_t n, int32_t m, int32_t vocab) {
    return n >= 1 && m >= 1 && m <= kMostDraft && vocab >= 1 && vocab <= (1 << 30) && n <= kMostRows && 2 * n * m <= kMostRows && 2 * n * m * row_blocks(vocab) <= kMostBlocks;
}

template <class T>
int launch_verify(const VerifyIn& in, hipStream_t stream) {
    const int64_t rows = in.n * in.m + (in.drafts ? in.n * (in.m - 1) : 0);
    constexpr int kWaves = kSumThreads / 64;
    hipLaunchKernelGGL((block_sums_kernel<T>), dim3((unsigned)((rows * in.row_blocks + kWaves - 1) / kWaves)), dim3(kSumThreads), 0, stream, in);
    HIP_TRY(hipGetLastError());
    if (!in.drafts) {
        hipLaunchKernelGGL((draw_rows_kernel<T>), dim3((unsigned)(in.n * in.m)), dim3(64), 0, stream, in);
        HIP_TRY(hipGetLastError());
        hipLaunchKernelGGL(verify_tree_kernel, dim3((unsigned)in.n), dim3(64), 0, stream, in);
        HIP_TRY(hipGetLastError());
        return IVFPQ_OK;
    }
    hipLaunchKernelGGL((verify_chain_kernel<T>), dim3((unsigned)in.n), dim3(kWalkThreads), 0, stream, in);
    HIP_TRY(hipGetLastError());
    // sequences of two rows at least, or nothing was drafted: fewer than 2^26 waves
    hipLaunchKernelGGL((left_sums_kernel<T>), dim3((unsigned)((in.n * in.left_blocks + kWaves - 1) / kWaves)), dim3(kSumThreads), 0, stream, in);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL((draw_left_kernel<T>), dim3((unsigned)in.n), dim3(64), 0, stream, in);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

}  // namespace

extern "C" {

size_t ivfpq_verify_drafts_workspace_bytes(int64_t n, int32_t m, int32_t vocab, int32_t with_drafts) {
    return verify_shape(n, m, vocab) ? verify_space(n, m, vocab, with_drafts != 0).bytes() : 0;
}

int ivfpq_verify_drafts(const void* d_logits, int32_t dtype, int64_t n, int32_t m, int32_t vocab, int64_t row_stride, const int32_t* d_tokens,
                        const int32_t* d_parents, const int32_t* d_counts, const float* d_uniforms, double temperature, const void* d_draft_logits,
                        int64_t draft_stride, const float* d_accept, int32_t* d_path, int32_t* d_kept, int32_t* d_next, float* d_logprobs,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded("ivfpq_verify_drafts", [&] {
        const char* what = "ivfpq_verify_drafts";
        if (!known_dtype(dtype)) return fail(IVFPQ_EINVAL, "%s: unknown dtype %d", what, dtype);
        if (n < 0 || m < 1 || vocab < 1) return fail(IVFPQ_EINVAL, "%s: bad shape (n=%lld m=%d vocab=%d)", what, (long long)n, m, vocab);
        if (m > kMostDraft) return fail(IVFPQ_EUNSUPPORTED, "%s: m=%d (limit %d rows)", what, m, kMostDraft);
        if (vocab > (1 << 30)) return fail(IVFPQ_EUNSUPPORTED, "%s: vocab=%d (limit 2^30)", what, vocab);
        if (!(temperature >= 1e-6 && temperature <= 1e6)) return fail(IVFPQ_EINVAL, "%s: temperature outside [1e-6, 1e6]", what);
        if (d_draft_logits && d_parents) return fail(IVFPQ_EINVAL, "%s: drafts that were drawn are a chain, without parents", what);
        if (n == 0) return (int)IVFPQ_OK;
        if (!verify_shape(n, m, vocab)) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld m=%d vocab=%d: over the limits (2^20 rows, 2^24 blocks of 2048 logits)", what, (long long)n, m, vocab);
        if (!d_logits || !d_tokens || !d_path || !d_kept || !d_next || !d_logprobs) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        if (d_draft_logits && (!d_uniforms || !d_accept)) return fail(IVFPQ_EINVAL, "%s: drafts that were drawn need both random numbers", what);
        if (n * m > 1 && row_stride < vocab) return fail(IVFPQ_EINVAL, "%s: row stride %lld below vocab=%d", what, (long long)row_stride, vocab);
        if (d_draft_logits && n * (m - 1) > 1 && draft_stride < vocab) return fail(IVFPQ_EINVAL, "%s: draft stride %lld below vocab=%d", what, (long long)draft_stride, vocab);
        if ((uintptr_t)d_logits % value_bytes(dtype) || (uintptr_t)d_draft_logits % value_bytes(dtype)) return fail(IVFPQ_EINVAL, "%s: logits are not aligned to their type", what);
        const bool drafts = d_draft_logits && m > 1;       // one row drafts nothing
        const VerifySpace space = verify_space(n, m, vocab, drafts);
        if (!d_workspace) return fail(IVFPQ_EINVAL, "%s: null workspace", what);
        if ((uintptr_t)d_workspace % kAlign) return fail(IVFPQ_EINVAL, "%s: workspace not aligned to %zu bytes", what, kAlign);
        if (workspace_bytes < space.bytes()) return fail(IVFPQ_ENOSPACE, "%s: workspace %zu bytes, need %zu", what, workspace_bytes, space.bytes());
        char* ws = (char*)d_workspace;
        const VerifyIn in{d_logits, drafts ? d_draft_logits : nullptr, row_stride, draft_stride, d_tokens, d_parents, d_counts, d_uniforms, d_accept,
                          (BlockSum*)ws, (double*)(ws + space.blocks), (Stop*)(ws + space.blocks + space.left), (Said*)(ws + space.blocks + space.left + space.stops), d_path, d_kept, d_next, d_logprobs, n, m, vocab,
                          row_blocks(vocab), left_blocks(vocab), 1.4426950408889634 / temperature};
        return with_value_type(dtype, [&](auto t) { return launch_verify<decltype(t)>(in, (hipStream_t)hip_stream); });
    });
}

}  // extern "C"
