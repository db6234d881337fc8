// Attention of drafted rows over a paged cache: ivfpq_draft_attention.
//
// For a row's query q, out = sum_p w_p v_p / sum_p w_p with w_p = 2^(s_p - r), s_p = scale log2(e) q . k_p and any reference r: one pass over the
// places, in which r follows the largest s only when that has left r far behind, and sums so far are scaled then.
//
// The rows of the heads that share keys are columns of two matrix products, S = K Q^T and O = V^T W^T, with 16 x 16 x 32 instructions: a tile is
// 32 places and 16 columns.  Keys are dealt to the rows of the first product so that its results are, lane by lane, the operand of the
// second (place 8 g + j of a tile is with lane group g in both), and the cache holds the values of 8 places side by side: nothing goes
// through the LDS between the cache and the sums.
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
    float* sums;                      // splits > 1: [n * m * heads][splits][d]
    float2* norms;                    // [n * m * heads][splits]: reference, sum of weights
    const int* parents;               // [n][m] or null
    long long q_stride, out_stride, n;
    int heads, blocks, splits;
    float scale;                      // with log2(e)
    Pages at;
};

constexpr int kAttentionThreads = 256, kTile = 32;
// A reference is the largest s of its time less kBelow, and follows when an s is more than kAhead over it: weights are up to 2^14 (fp16 holds
// 65,504), and those under 2^-24 of the largest, which fp16 would cut off, are kept down to 2^-30.
constexpr float kBelow = 6.f, kAhead = 14.f;

// T: type of the cache.  KC: 32 components of a head each (d <= 32 KC; EXACT: equal).  NQ: tiles of 16 columns a wave.  APART: a wave has columns of its
// own and goes over all places of the workgroup; otherwise the four waves share their columns, take every fourth tile, and add up at the end.
template <class T, int KC, int NQ, bool APART, bool EXACT>
__global__ __launch_bounds__(kAttentionThreads) void attention_kernel(AttentionIn in) {
    constexpr int VT = KC * 2;                       // tiles of 16 components
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, group = lane >> 4;
    const int d = EXACT ? KC * 32 : in.at.d;
    const int shift = in.at.shift, in_page = in.at.page() - 1;

    // blocks of columns that read the same places are 8 workgroups apart: on one XCD, whose L2 they share
    const unsigned order = blockIdx.x, turn = order / 8;
    const int block = (int)(turn % in.blocks);
    const long long pass = (long long)(turn / in.blocks) * 8 + order % 8;      // (split, head, sequence)
    if (pass >= in.n * in.at.kv_heads * in.splits) return;
    const long long s = pass % in.n;
    const int head = (int)(pass / in.n % in.at.kv_heads), split = (int)(pass / in.n / in.at.kv_heads);
    const int share = in.heads / in.at.kv_heads;     // heads that share keys
    const int len = in.at.len(s), count = in.at.count(s), m = in.at.m;
    const int first_col = (block * (APART ? 4 : 1) + (APART ? wave : 0)) * NQ * 16;
    const int all_cols = m * share, used_cols = count * share;

    // what each column sees of the rows: bits of a tree, or the rows up to its own
    uint64_t line = 0;
    if (in.parents) {
        int up = -1;
        if (lane < count) {
            up = in.parents[s * m + lane];
            if (up < 0 || up >= lane) up = -1;
            line = (uint64_t)1 << lane;
        }
        for (int far = 1; far < 64; far *= 2) {      // a row has up to 63 ancestors
            const uint64_t above = __shfl((unsigned long long)line, max(up, 0));
            const int next = __shfl(up, max(up, 0));
            if (up >= 0) {
                line |= above;
                up = next;
            }
        }
    }
    u32x4 q[NQ][KC];
    int row[NQ];
    uint64_t sees[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        const int x = first_col + t * 16 + col;
        row[t] = x < used_cols ? x / share : -1;     // -1: nothing to do in this column
        sees[t] = __shfl((unsigned long long)line, max(row[t], 0) & 63);
        const T* from = (const T*)in.q + (s * m + max(row[t], 0)) * in.q_stride + (long long)(head * share + x % share) * d + group * 8;
#pragma unroll
        for (int c = 0; c < KC; ++c) q[t][c] = row[t] >= 0 && (EXACT || c * 32 + group * 8 < d) ? *reinterpret_cast<const u32x4*>(from + c * 32) : u32x4{};
    }
    f32x4 sums[NQ][VT];
    float reference[NQ], total[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        reference[t] = -INFINITY;
        total[t] = 0.f;
#pragma unroll
        for (int v = 0; v < VT; ++v) sums[t][v] = f32x4{};
    }

    // tiles of the workgroup: of the places up to the last that one of its columns sees
    const int block_cols = NQ * 16 * (APART ? 4 : 1);
    const int last_col = min((block + 1) * block_cols, used_cols) - 1;
    const bool nothing = block * block_cols >= used_cols;
    const long long places = nothing ? 0 : in.parents ? (long long)len + count : (long long)len + last_col / share + 1;
    const int tiles = (int)min((places + kTile - 1) / kTile, (((long long)in.at.most << shift) + kTile - 1) / kTile);
    constexpr int STEP = APART ? 1 : 4;
    int each = (tiles + in.splits - 1) / in.splits;
    each = (each + STEP - 1) / STEP * STEP;
    const int first = (int)min((long long)split * each, (long long)tiles), end = min(first + each, tiles);
    const int* pages = in.at.pages + s * in.at.stride;

    const long long page_values = in.at.page_values();
    const int key_in_tile = (col >> 2) * 8 + (col & 3);             // and 4 more in the second half of S
    const bool second_k = col >> 3, second_v = group >> 1;          // in the tile's second 16 places
    const int k_lane = (key_in_tile & 15) * d + group * 8, v_lane = (group & 1) * 8 * d + col * 8;
    const T* const k_head = (const T*)in.k_cache + ((long long)head << shift) * d;
    const T* const v_head = (const T*)in.v_cache + ((long long)head << shift) * d;

    // The pages of a tile's two halves; one that is not there is read as page 0 (there is one: without pages there are no tiles), and the tile is
    // gone over with a mask.
    const auto find = [&](int tile, int& p0, int& p1) {
        const long long at = (long long)tile * kTile, i0 = at >> shift, i1 = (at + 16) >> shift;
        p0 = tile < end && i0 < in.at.most ? pages[i0] : -1;
        p1 = tile < end && i1 < in.at.most ? pages[i1] : -1;
        if (p0 >= in.at.n_pages) p0 = -1;
        if (p1 >= in.at.n_pages) p1 = -1;
    };
    u32x4 keys[2][KC], values[VT];
    const auto load_keys = [&](int tile, int p0, int p1) {
        const int off0 = (tile * kTile) & in_page, off1 = (tile * kTile + 16) & in_page;
        const T* from = k_head + (second_k ? max(p1, 0) * page_values + off1 * d : max(p0, 0) * page_values + off0 * d) + k_lane;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < KC; ++c) keys[t][c] = EXACT || c * 32 + group * 8 < d ? *reinterpret_cast<const u32x4*>(from + t * 4 * d + c * 32) : u32x4{};
    };
    const auto load_values = [&](int tile, int p0, int p1) {
        const int off0 = (tile * kTile) & in_page, off1 = (tile * kTile + 16) & in_page;
        const T* from = v_head + (second_v ? max(p1, 0) * page_values + off1 * d : max(p0, 0) * page_values + off0 * d) + v_lane;
#pragma unroll
        for (int v = 0; v < VT; ++v) values[v] = EXACT || v * 16 + col < d ? *reinterpret_cast<const u32x4*>(from + v * 128) : u32x4{};
    };

    int tile = first + (APART ? 0 : wave);
    int page0 = -1, page1 = -1, next0 = -1, next1 = -1;
    find(tile, page0, page1);
    find(tile + STEP, next0, next1);
    if (tile < end) {
        load_keys(tile, page0, page1);
        load_values(tile, page0, page1);
    }
    // One tile; the next one's keys are loaded as soon as this one's are used, and its values likewise.
    const auto go = [&](auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        int after0, after1;
        find(tile + 2 * STEP, after0, after1);
        const bool more = tile + STEP < end;
        f32x4 score[NQ][2];
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 acc{};
#pragma unroll
                for (int c = 0; c < KC; ++c) acc = multiply<T>(keys[h][c], q[t][c], acc);
                score[t][h] = acc;
            }
        if (more) load_keys(tile + STEP, next0, next1);

        // weights in the order of the places 8 group + j; one that a column does not see is 0
        const int first_place = tile * kTile + group * 8;
        const bool there = second_v ? page1 >= 0 : page0 >= 0;       // the page of this lane's places
        u32x4 weights[NQ];
        unsigned hidden[NQ];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            float w[8];
            hidden[t] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = score[t][j >> 2][j & 3] * in.scale;
            if constexpr (MASKED) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int behind = first_place + j - len;        // row whose place it is
                    const bool drafted = in.parents ? behind < 64 && (sees[t] >> (behind & 63) & 1) : behind <= row[t];
                    if (!(there && row[t] >= 0 && (behind < 0 || drafted))) {
                        w[j] = -INFINITY;
                        hidden[t] |= 1u << j;
                    }
                }
            }
            float most = max3(max3(w[0], w[1], w[2]), max3(w[3], w[4], w[5]), fmaxf(w[6], w[7]));
            if (__any(most > reference[t] + kAhead)) {
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                const float now = fmaxf(reference[t], most - kBelow);
                const float shrink = now == reference[t] ? 1.f : exp2_fast(reference[t] - now);
                reference[t] = now;
                total[t] *= shrink;
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] *= shrink;
            }
            const float r = reference[t] == -INFINITY ? 0.f : reference[t];      // nothing seen so far
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = exp2_fast(w[j] - r);
            total[t] += tree_sum<8>(w);
            weights[t] = narrow8<T>(w);
        }

        if constexpr (!MASKED) {
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] = multiply<T>(values[v], weights[t], sums[t][v]);
        } else {
            // 0 times infinity is no number, so values that not every column sees must not meet weights of 0: those of places without a row go, and
            // infinities and NaNs of rows are added to the columns that see them, place by place
            constexpr uint32_t kOnes = std::is_same<T, half_t>::value ? 0x7C00u : 0x7F80u;
            const auto wild = [&](uint32_t x) {       // the halves of a word that are infinities or NaNs
                return ((x & kOnes) == kOnes ? 0xFFFFu : 0u) | ((x & kOnes << 16) == kOnes << 16 ? 0xFFFF0000u : 0u);
            };
            uint32_t odd[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t holds = (there && first_place + 2 * i < places ? 0xFFFFu : 0u) | (there && first_place + 2 * i + 1 < places ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int v = 0; v < VT; ++v) {
                    values[v][i] &= holds;
                    odd[i] |= wild(values[v][i]);
                }
            }
            if (__any((odd[0] | odd[1] | odd[2] | odd[3]) != 0)) {
#pragma unroll 1
                for (int place = 0; place < kTile; ++place) {
                    const int g = place >> 3, j = place & 7;
                    const uint32_t field = 0xFFFFu << (j & 1) * 16, mine = j < 2 ? odd[0] : j < 4 ? odd[1] : j < 6 ? odd[2] : odd[3];
                    if (!__any(group == g && (mine & field))) continue;
                    bool seen[NQ];
#pragma unroll
                    for (int t = 0; t < NQ; ++t) seen[t] = row[t] >= 0 && !(__shfl(hidden[t], g * 16 + col) >> j & 1);
#pragma unroll
                    for (int v = 0; v < VT; ++v) {
                        u32x4 one;                   // this place's values, where they are odd
#pragma unroll
                        for (int i = 0; i < 4; ++i) one[i] = group == g && i == j >> 1 ? values[v][i] & field & wild(values[v][i]) : 0u;
#pragma unroll
                        for (int t = 0; t < NQ; ++t) {
                            const f32x4 with = multiply<T>(one, weights[t], sums[t][v]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) sums[t][v][i] = seen[t] ? with[i] : sums[t][v][i];
                        }
                    }
                }
#pragma unroll
                for (int v = 0; v < VT; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) values[v][i] &= ~wild(values[v][i]);
            }
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] = multiply<T>(values[v], weights[t], sums[t][v]);
        }
        if (more) load_values(tile + STEP, next0, next1);
        page0 = next0, page1 = next1;
        next0 = after0, next1 = after1;
        tile += STEP;
    };
    // tiles of places that every column sees, then those with rows, or (seldom) all from the first that lacks a page
    const int seen_by_all = min(end, len / kTile);
    while (tile < seen_by_all && page0 >= 0 && page1 >= 0) go(std::false_type{});
    while (tile < end) go(std::true_type{});

    // a column's lanes hold sums of all its places, but each the total of its own 8 of every 32
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        total[t] += __shfl_xor(total[t], 16);
        total[t] += __shfl_xor(total[t], 32);
        if (row[t] < 0) {                            // went along with the others over the tiles without a mask
            total[t] = 0.f;
            reference[t] = -INFINITY;
#pragma unroll
            for (int v = 0; v < VT; ++v) sums[t][v] = f32x4{};
        }
    }
    if constexpr (!APART) {
        // the waves' sums about the largest of their references, added up in a fixed order: 0 + 2, 1 + 3, then both
        __shared__ float refs[4][NQ][16], totals[4][NQ][16];
        __shared__ f32x4 shared[2][NQ][VT][64];
        if (group == 0)
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                refs[wave][t][col] = reference[t];
                totals[wave][t][col] = total[t];
            }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            float most = -INFINITY, sum = 0.f;
            for (int w = 0; w < 4; ++w) most = fmaxf(most, refs[w][t][col]);
            for (int w = 0; w < 4; ++w) sum += refs[w][t][col] == -INFINITY ? totals[w][t][col] : totals[w][t][col] * (refs[w][t][col] == most ? 1.f : exp2_fast(refs[w][t][col] - most));
            const float shrink = reference[t] == most || reference[t] == -INFINITY ? 1.f : exp2_fast(reference[t] - most);
#pragma unroll
            for (int v = 0; v < VT; ++v) sums[t][v] *= shrink;
            reference[t] = most;
            total[t] = sum;
        }
        if (wave >= 2)
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) shared[wave - 2][t][v][lane] = sums[t][v];
        __syncthreads();
        if (wave < 2)
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) sums[t][v] += shared[wave][t][v][lane];
        __syncthreads();
        if (wave == 1)
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int v = 0; v < VT; ++v) shared[0][t][v][lane] = sums[t][v];
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int t = 0; t < NQ; ++t)
#pragma unroll
            for (int v = 0; v < VT; ++v) sums[t][v] += shared[0][t][v][lane];
    }

#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        const int x = first_col + t * 16 + col;
        if (x >= all_cols) continue;
        const int h = head * share + x % share;
        const long long flat = s * m + x / share;
        if (in.splits > 1) {
            const long long at = (flat * in.heads + h) * in.splits + split;
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

// The parts of a row and head added up: a thread has 4 components of one of them.
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionIn in, long long pieces) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int d = in.at.d, per = d / 4;
    const long long at = i / per;                    // row and head
    const int c = (int)(i % per) * 4;
    float most = -INFINITY;
    for (int p = 0; p < in.splits; ++p) most = fmaxf(most, in.norms[at * in.splits + p].x);
    f32x4 sum{};
    float total = 0.f;
    for (int p = 0; p < in.splits; ++p) {
        const float2 norm = in.norms[at * in.splits + p];
        const float by = norm.x == most || norm.x == -INFINITY ? 1.f : exp2_fast(norm.x - most);
        total += norm.y * by;
        sum += *reinterpret_cast<const f32x4*>(in.sums + (at * in.splits + p) * d + c) * by;
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
    const long long row = at / in.heads;
    const int h = (int)(at % in.heads);
    if (in.lse && c == 0) in.lse[at] = total == 0.f ? -INFINITY : (most + __log2f(total)) * kLn2;
    typedef T v4 __attribute__((ext_vector_type(4)));
    v4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (T)(sum[j] * by);
    *reinterpret_cast<v4*>((T*)in.out + row * in.out_stride + (long long)h * d + c) = y;
}

template <class T, int KC, bool EXACT>
int launch_attention(const AttentionIn& in, const AttentionPlan& plan, hipStream_t stream) {
    const long long passes = in.n * in.at.kv_heads * in.splits;
    const dim3 grid((unsigned)((passes + 7) / 8 * 8 * in.blocks)), threads(kAttentionThreads);
    constexpr int MOST = KC > 4 ? 2 : 4;
    if (plan.apart) hipLaunchKernelGGL((attention_kernel<T, KC, MOST, true, EXACT>), grid, threads, 0, stream, in);
    else if (plan.tiles == 1) hipLaunchKernelGGL((attention_kernel<T, KC, 1, false, EXACT>), grid, threads, 0, stream, in);
    else if (plan.tiles == 2) hipLaunchKernelGGL((attention_kernel<T, KC, 2, false, EXACT>), grid, threads, 0, stream, in);
    else if constexpr (MOST == 4) hipLaunchKernelGGL((attention_kernel<T, KC, 4, false, EXACT>), grid, threads, 0, stream, in);
    HIP_TRY(hipGetLastError());
    if (in.splits > 1) {
        const long long pieces = in.n * in.at.m * in.heads * (in.at.d / 4);
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, stream, in, pieces);
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
bool fits_launch(int64_t n, int32_t kv_heads, const AttentionPlan& plan) { return n * kv_heads * plan.splits * plan.blocks <= ((int64_t)1 << 23); }

}  // namespace

extern "C" {

size_t ivfpq_draft_attention_workspace_bytes(int64_t n, int32_t m, int32_t heads, int32_t kv_heads, int32_t d, int64_t max_places) {
    if (!known_shape(n, m, heads, kv_heads, d, max_places)) return 0;
    const AttentionPlan plan = attention_plan(n, m, heads, kv_heads, d, max_places);
    return align_up((size_t)attention_split_floats(n, m, heads, d, plan.splits) * sizeof(float));
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
        const AttentionPlan plan = attention_plan(n, m, heads, kv_heads, d, max_places);
        if (!fits_launch(n, kv_heads, plan)) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld m=%d heads=%d kv_heads=%d: over 2^23 workgroups", what, (long long)n, m, heads, kv_heads);
        const size_t need = align_up((size_t)attention_split_floats(n, m, heads, d, plan.splits) * sizeof(float));
        if (need) {
            if (!d_workspace) return fail(IVFPQ_EINVAL, "%s: null workspace", what);
            if ((uintptr_t)d_workspace % kAlign) return fail(IVFPQ_EINVAL, "%s: workspace not aligned to %zu bytes", what, kAlign);
            if (workspace_bytes < need) return fail(IVFPQ_ENOSPACE, "%s: workspace %zu bytes, need %zu", what, workspace_bytes, need);
        }
        AttentionIn in{d_q, d_k_cache, d_v_cache, d_out, d_lse, (float*)d_workspace, nullptr, d_parents, q_stride, out_stride, n, heads, plan.blocks, plan.splits,
                       (float)((double)scale * 1.4426950408889634), pages_in(d_pages, max_pages, d_lens, d_counts, n_pages, kv_heads, page, d, m)};
        in.norms = (float2*)(in.sums + (size_t)rows * heads * plan.splits * d);      // d is a multiple of 8
        // max_places bounds what is looked at: the table's end does
        in.at.most = n_pages ? (int)std::min<int64_t>(max_pages, (max_places + page - 1) / page) : 0;
        return with_value_type(cache_dtype, [&](auto t) {
            using T = decltype(t);
            if constexpr (sizeof(T) == 4) return (int)IVFPQ_EINVAL;
            else return launch_attention<T>(in, plan, (hipStream_t)hip_stream);
        });
    });
}

}  // extern "C"
