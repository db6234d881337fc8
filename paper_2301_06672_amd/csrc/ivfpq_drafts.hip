// Search results as trees of drafted tokens: what ivfpq_neighbour_drafts does.
//
// The continuations of a query's neighbours share beginnings; a node of the tree is a beginning, its weight the sum of theirs.  Weights are whole
// numbers of 2^-32, so sums are the same in any order and a node never weighs more than its parent: with ties given to the
// shallower node, the heaviest nodes are a tree, and every one comes behind its parent.  A node is named by its depth t and the first neighbour j
// that runs through it; its key, (weight, 14 - t, 1023 - j) from the top bit down, has the order wanted and differs from all others.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_hip_util.hpp"
#include "ivfpq_values.hpp"

using namespace ivfpq;

namespace {

struct DraftsIn {
    const long long* ids;             // [nq][k]
    const float* dists;
    const int* text;                  // [n_ids]
    const int* last;                  // [nq]
    long long n_ids;
    double temperature;
    int k, depth, m;
};
struct DraftsOut {
    int *tokens, *parents, *depths, *counts;
    float* logprobs;
};

constexpr int kMostNodes = IVFPQ_MAX_DRAFT - 1;
typedef unsigned long long u64;

// One workgroup a query; K: room for neighbours.  What bounds it is latency: 1,024 queries of 100 neighbours, 10 tokens deep, 36 us (86 with a token a level read
// when it is needed and a search for the smallest key in the LDS; 41 with two waves a query), one query of 32 neighbours, 6 deep, 15 us.  A level of the tree at a time: the neighbours that went one way so far and go on with
// the same token meet in a slot of a hash table in the LDS, which gives their node its first neighbour and its weight.  Nodes collect in
// a list; when that is full, all but the m - 1 largest keys go, and neighbours whose node went follow no further.
template <int THREADS, int K>
__global__ __launch_bounds__(THREADS) void neighbour_drafts_kernel(DraftsIn in, DraftsOut out) {
    constexpr int EACH = K / THREADS, WAVES = THREADS / 64, SLOTS = 2 * K;       // at most half full
    constexpr int ROOM = K <= 256 ? 512 : 2048;                                  // over kMostNodes + K
    constexpr u64 kFree = ~0ull;
    __shared__ u64 slots[SLOTS], weights[SLOTS];                                 // (group, token), sum of weights
    __shared__ int first_of[SLOTS];
    __shared__ u64 keys[ROOM];
    __shared__ int tokens[ROOM], parents[ROOM];                                  // a parent: the low 14 bits of its key, or -1
    __shared__ u64 best_keys[kMostNodes];
    __shared__ int best_tokens[kMostNodes], best_parents[kMostNodes], names[kMostNodes];
    __shared__ int texts[IVFPQ_MAX_DRAFT_DEPTH][K];
    __shared__ int listed, counts[3];
    __shared__ u64 sums[WAVES];
    __shared__ float scratch[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, k = in.k, nodes = in.m - 1;
    const long long q = blockIdx.x;

    int token[EACH], group[EACH];
    u64 weight[EACH];                  // 0: follows no further
    float dist[EACH];
    float nearest = INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = i * THREADS + tid;
        dist[i] = INFINITY;
        token[i] = -1;
        if (j < k) {
            const long long id = in.ids[q * k + j];
            const float d = in.dists[q * k + j];
            if (id >= 0 && id < in.n_ids && fabsf(d) < INFINITY) {
                // the whole continuation, so that the way down waits for memory once
                int words[IVFPQ_MAX_DRAFT_DEPTH];
#pragma unroll
                for (int t = 0; t < IVFPQ_MAX_DRAFT_DEPTH; ++t) words[t] = t < in.depth && id + t < in.n_ids ? in.text[id + t] : -1;
#pragma unroll
                for (int t = 1; t < IVFPQ_MAX_DRAFT_DEPTH; ++t) texts[t][j] = words[t];
                token[i] = words[0];
                if (token[i] >= 0) dist[i] = d;
            }
        }
        nearest = fminf(nearest, dist[i]);
    }
    if (tid == 0) listed = 0;
    nearest = -block_max<THREADS>(-nearest, scratch);
    u64 total = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        group[i] = 0;
        weight[i] = dist[i] < INFINITY ? (u64)rint(exp(((double)nearest - (double)dist[i]) / in.temperature) * 0x1p32) : 0;
        total += weight[i];
    }
    total = block_sum<THREADS>(total, sums);

    // Keeps the `nodes` largest keys of the list, in any order; -> a number that so many keys are not under.  Bit by bit from the top, until the
    // number parts the keys.
    const auto prune = [&] {
        constexpr int HELD = ROOM / THREADS;
        const int n = listed;
        u64 mine[HELD];
#pragma unroll
        for (int i = 0; i < HELD; ++i) mine[i] = i * THREADS + tid < n ? keys[i * THREADS + tid] : 0;
        u64 least = 0;
        if (tid < 3) counts[tid] = 0;
        __syncthreads();
        int round = 0;
        for (int bit = 56; bit >= 0; --bit) {
            const u64 probe = least | 1ull << bit;
            int over = 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i) over += __popcll(__ballot(mine[i] >= probe));
            if constexpr (WAVES > 1) {               // counts of three rounds: one is added up, one read, one cleared for the next
                if (lane == 0) atomicAdd(&counts[round], over);
                if (tid == 0) counts[round == 2 ? 0 : round + 1] = 0;
                __syncthreads();
                over = counts[round];
                round = round == 2 ? 0 : round + 1;
            }
            if (over >= nodes) least = probe;
            if (over == nodes) break;
        }
        __syncthreads();
        if (tid == 0) listed = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (mine[i] >= least && mine[i] != 0) {
                const int to = atomicAdd(&listed, 1);
                best_keys[to] = mine[i];
                best_tokens[to] = tokens[i * THREADS + tid];
                best_parents[to] = parents[i * THREADS + tid];
            }
        __syncthreads();
        for (int i = tid; i < listed; i += THREADS) {
            keys[i] = best_keys[i];
            tokens[i] = best_tokens[i];
            parents[i] = best_parents[i];
        }
        __syncthreads();
        return least;
    };

    for (int i = tid; i < SLOTS; i += THREADS) {
        slots[i] = kFree;
        weights[i] = 0;
        first_of[i] = K;
    }
    u64 least = 0;
    for (int t = 0; t < in.depth && nodes > 0; ++t) {
        bool going = false;
#pragma unroll
        for (int i = 0; i < EACH; ++i) going |= weight[i] != 0;
        if (!__syncthreads_or(going)) break;         // and the table is free behind it
        int slot[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            slot[i] = -1;
            if (!weight[i]) continue;
            const u64 name = (u64)group[i] << 32 | (unsigned)token[i];
            unsigned here = ((unsigned)token[i] * 2654435761u + (unsigned)group[i] * 2246822519u) >> 16 & (SLOTS - 1);
            for (;;) {                               // ends: more slots than neighbours
                const u64 held = atomicCAS(&slots[here], kFree, name);
                if (held == kFree || held == name) break;
                here = (here + 1) & (SLOTS - 1);
            }
            slot[i] = (int)here;
            atomicMin(&first_of[here], i * THREADS + tid);
            atomicAdd(&weights[here], weight[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (!weight[i]) continue;
            const int j = first_of[slot[i]];
            const u64 key = weights[slot[i]] << 14 | (unsigned)(14 - t) << 10 | (unsigned)(1023 - j);
            if (key < least) {                       // not among the largest, nor is anything behind it
                weight[i] = 0;
                continue;
            }
            if (j == i * THREADS + tid) {
                const int to = atomicAdd(&listed, 1);
                keys[to] = key;
                tokens[to] = token[i];
                parents[to] = t == 0 ? -1 : (15 - t) << 10 | (1023 - group[i]);
            }
            group[i] = j;
        }
        __syncthreads();
        if (listed > ROOM - K) least = prune();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (slot[i] >= 0) {                      // the level's slots are free again: those who took them know
                slots[slot[i]] = kFree;
                weights[slot[i]] = 0;
                first_of[slot[i]] = K;
            }
            token[i] = weight[i] && t + 1 < in.depth ? texts[t + 1][i * THREADS + tid] : -1;
            if (token[i] < 0) weight[i] = 0;
        }
    }
    __syncthreads();
    if (listed > nodes) prune();

    // in order: a node's row is the number of keys over its own, behind row 0
    const int n = listed;
    int row = 0;
    u64 key = 0;
    if (tid < n) {
        key = keys[tid];
        row = 1;
        for (int i = 0; i < n; ++i) row += keys[i] > key;
        names[row - 1] = (int)(key & 0x3FFF);
    }
    __syncthreads();
    const long long base = q * in.m;
    if (tid < n) {
        const int up = parents[tid];
        int parent = 0;
        for (int i = 0; i < n; ++i) parent = up >= 0 && names[i] == up ? i + 1 : parent;
        out.tokens[base + row] = tokens[tid];
        out.parents[base + row] = parent;
        out.depths[base + row] = 15 - (int)(key >> 10 & 15);
        out.logprobs[base + row] = (float)log((double)(key >> 14) / (double)total);
    }
    if (tid == 0) {
        out.tokens[base] = in.last[q];
        out.parents[base] = -1;
        out.depths[base] = 0;
        out.logprobs[base] = 0.f;
        out.counts[q] = 1 + n;
    }
    for (int i = 1 + n + tid; i < in.m; i += THREADS) {
        out.tokens[base + i] = -1;
        out.parents[base + i] = -1;
        out.depths[base + i] = 0;
        out.logprobs[base + i] = -INFINITY;
    }
}

}  // namespace

extern "C" int ivfpq_neighbour_drafts(const int64_t* d_ids, const float* d_dists, int64_t nq, int32_t k, const int32_t* d_text, int64_t n_ids,
                                      const int32_t* d_last, double temperature, int32_t depth, int32_t m, int32_t* d_tokens,
                                      int32_t* d_parents, int32_t* d_depths, float* d_logprobs, int32_t* d_counts, void* hip_stream) {
    return guarded("ivfpq_neighbour_drafts", [&] {
        const char* what = "ivfpq_neighbour_drafts";
        if (nq < 0 || n_ids < 0) return fail(IVFPQ_EINVAL, "%s: bad shape", what);
        if (k < 1 || k > IVFPQ_MAX_LISTED) return fail(IVFPQ_EINVAL, "%s: k=%d outside [1, %d]", what, k, (int)IVFPQ_MAX_LISTED);
        if (depth < 1 || depth > IVFPQ_MAX_DRAFT_DEPTH) return fail(IVFPQ_EINVAL, "%s: depth=%d outside [1, %d]", what, depth, (int)IVFPQ_MAX_DRAFT_DEPTH);
        if (m < 1 || m > IVFPQ_MAX_DRAFT) return fail(IVFPQ_EINVAL, "%s: m=%d outside [1, %d]", what, m, (int)IVFPQ_MAX_DRAFT);
        if (!(temperature >= 1e-30 && temperature <= 1e30)) return fail(IVFPQ_EINVAL, "%s: temperature outside [1e-30, 1e30]", what);
        if (nq == 0) return (int)IVFPQ_OK;
        if (!d_ids || !d_dists || !d_last || !d_tokens || !d_parents || !d_depths || !d_logprobs || !d_counts || (n_ids > 0 && !d_text))
            return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        const hipStream_t stream = (hipStream_t)hip_stream;
        constexpr int64_t kPiece = 1 << 22;                // a launch has fewer than 2^32 threads
        for (int64_t at = 0; at < nq; at += kPiece) {
            const DraftsIn in{(const long long*)d_ids + at * k, d_dists + at * k, d_text, d_last + at, (long long)n_ids, temperature, k, depth, m};
            const DraftsOut out{d_tokens + at * m, d_parents + at * m, d_depths + at * m, d_counts + at, d_logprobs + at * m};
            const dim3 grid((unsigned)std::min(kPiece, nq - at));
            if (k <= 64) hipLaunchKernelGGL((neighbour_drafts_kernel<64, 64>), grid, dim3(64), 0, stream, in, out);
            else if (k <= 128) hipLaunchKernelGGL((neighbour_drafts_kernel<64, 128>), grid, dim3(64), 0, stream, in, out);
            else if (k <= 256) hipLaunchKernelGGL((neighbour_drafts_kernel<256, 256>), grid, dim3(256), 0, stream, in, out);
            else hipLaunchKernelGGL((neighbour_drafts_kernel<256, 1024>), grid, dim3(256), 0, stream, in, out);
            HIP_TRY(hipGetLastError());
        }
        return (int)IVFPQ_OK;
    });
}
