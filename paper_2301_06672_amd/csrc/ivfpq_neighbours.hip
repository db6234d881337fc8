// Search results as a distribution over tokens: what ivfpq_neighbour_tokens does.
//
// With t_j = (d_min - d_j) log2(e) / T the weight of neighbour j is 2^t_j; the neighbours that share a token add up at the
// first of them.  A query's tokens are in a hash table in the LDS, so the work goes with k.  A token's weights are taken about its
// nearest neighbour and added as whole numbers of 2^-53 (the largest is 1, at most 1024 are added): exact to 2^-43 of the
// sum, and the same in any order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_hip_util.hpp"
#include "ivfpq_values.hpp"

using namespace ivfpq;

namespace {

struct NeighboursIn {
    const long long* ids;             // [nq][k]
    const float* dists;
    const int* id_tokens;             // [n_ids]
    long long n_ids;
    float scale;                      // log2(e) / T
    int k;
};

// One workgroup a query; K: room for neighbours.  What bounds it is latency: ids, then tokens gathered from anywhere, then the table's
// atomics.  10,000 queries of 100 neighbours, tokens in a table of 40 MB: 23 us (24 MB and 10^6 sectors; 46 with every neighbour compared
// with every other), of 1,024 neighbours 198 us.
template <int THREADS, int K>
__global__ __launch_bounds__(THREADS) void neighbour_tokens_kernel(NeighboursIn in, int* __restrict__ tokens, float* __restrict__ logprobs) {
    constexpr int EACH = K / THREADS, WAVES = THREADS / 64, SLOTS = 2 * K;      // at most half full
    __shared__ unsigned long long sums[SLOTS];
    __shared__ int keys[SLOTS], first_of[SLOTS], near_of[SLOTS];               // near_of: the bits of the smallest -t
    __shared__ float scratch[WAVES];
    __shared__ int firsts[EACH * WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = in.k;
    const long long q = blockIdx.x;
    int mine[EACH];
    float dist[EACH];
    float nearest = INFINITY;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = i * THREADS + tid;
        mine[i] = -1;
        dist[i] = INFINITY;
        if (j < k) {
            const long long id = in.ids[q * k + j];
            const float d = in.dists[q * k + j];
            if (id >= 0 && id < in.n_ids && fabsf(d) < INFINITY) {
                mine[i] = in.id_tokens[id];
                if (mine[i] >= 0) dist[i] = d;
                else mine[i] = -1;
            }
        }
        nearest = fminf(nearest, dist[i]);
    }
    for (int i = tid; i < SLOTS; i += THREADS) {
        keys[i] = -1;
        first_of[i] = K;
        near_of[i] = 0x7FFFFFFF;
        sums[i] = 0;
    }
    nearest = -block_max<THREADS>(-nearest, scratch);      // and barriers behind the cleared table
    float total = 0.f;
    float far[EACH];                                       // -t
    int slot[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        far[i] = 0.f;
        slot[i] = 0;
        if (mine[i] < 0) continue;
        far[i] = fabsf((nearest - dist[i]) * in.scale);
        total += exp2_fast(-far[i]);
        unsigned at = ((unsigned)mine[i] * 2654435761u) >> 16 & (SLOTS - 1);
        for (;;) {                                         // ends: more slots than tokens
            const int held = atomicCAS(&keys[at], -1, mine[i]);
            if (held == -1 || held == mine[i]) break;
            at = (at + 1) & (SLOTS - 1);
        }
        slot[i] = (int)at;
        atomicMin(&first_of[at], i * THREADS + tid);
        atomicMin(&near_of[at], __float_as_int(far[i]));   // numbers that are not negative: their bits have their order
    }
    const float log_total = logf(block_sum<THREADS>(total, scratch));      // and barriers behind the filled table

#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (mine[i] >= 0) {
            const float near = __int_as_float(near_of[slot[i]]);
            if (near < INFINITY) atomicAdd(&sums[slot[i]], (unsigned long long)(exp2_fast(near - far[i]) * 0x1p53f));
        }
    __syncthreads();
    float logp[EACH];
    bool first[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        first[i] = mine[i] >= 0 && first_of[slot[i]] == i * THREADS + tid;
        logp[i] = 0.f;
        if (!first[i]) continue;
        const float near = __int_as_float(near_of[slot[i]]);
        // -inf: over 10^38 temperatures away
        logp[i] = near == INFINITY ? -INFINITY : logf((float)sums[slot[i]] * 0x1p-53f) - near * kLn2 - log_total;
    }
    // places: the distinct tokens before this one
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint64_t mask = __ballot(first[i]);
        if (lane == 0) firsts[i * WAVES + wave] = __popcll(mask);
    }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) {
                const uint64_t mask = __ballot(first[i]);
                if (first[i]) {
                    const int at = before + __popcll(mask & (((uint64_t)1 << lane) - 1));
                    tokens[q * k + at] = mine[i];
                    logprobs[q * k + at] = logp[i];
                }
            }
            before += firsts[i * WAVES + w];
        }
    for (int j = before + tid; j < k; j += THREADS) {
        tokens[q * k + j] = -1;
        logprobs[q * k + j] = -INFINITY;
    }
}

}  // namespace

extern "C" int ivfpq_neighbour_tokens(const int64_t* d_ids, const float* d_dists, int64_t nq, int32_t k, const int32_t* d_id_tokens,
                                      int64_t n_ids, float temperature, int32_t* d_tokens, float* d_logprobs, void* hip_stream) {
    return guarded("ivfpq_neighbour_tokens", [&] {
        const char* what = "ivfpq_neighbour_tokens";
        if (nq < 0 || n_ids < 0) return fail(IVFPQ_EINVAL, "%s: bad shape", what);
        if (k < 1 || k > IVFPQ_MAX_LISTED) return fail(IVFPQ_EINVAL, "%s: k=%d outside [1, %d]", what, k, (int)IVFPQ_MAX_LISTED);
        if (!(temperature >= 1e-30f && temperature <= 1e30f)) return fail(IVFPQ_EINVAL, "%s: temperature outside [1e-30, 1e30]", what);
        if (nq == 0) return (int)IVFPQ_OK;
        if (!d_ids || !d_dists || !d_tokens || !d_logprobs || (n_ids > 0 && !d_id_tokens)) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        const hipStream_t stream = (hipStream_t)hip_stream;
        constexpr int64_t kPiece = 1 << 22;                // a launch has fewer than 2^32 threads
        for (int64_t at = 0; at < nq; at += kPiece) {
            const NeighboursIn in{(const long long*)d_ids + at * k, d_dists + at * k, d_id_tokens, (long long)n_ids,
                                  (float)(1.4426950408889634 / (double)temperature), k};
            int* tokens = d_tokens + at * k;
            float* logprobs = d_logprobs + at * k;
            const dim3 grid((unsigned)std::min(kPiece, nq - at));
            if (k <= 64) hipLaunchKernelGGL((neighbour_tokens_kernel<64, 64>), grid, dim3(64), 0, stream, in, tokens, logprobs);
            else if (k <= 128) hipLaunchKernelGGL((neighbour_tokens_kernel<64, 128>), grid, dim3(64), 0, stream, in, tokens, logprobs);
            else if (k <= 256) hipLaunchKernelGGL((neighbour_tokens_kernel<256, 256>), grid, dim3(256), 0, stream, in, tokens, logprobs);
            else hipLaunchKernelGGL((neighbour_tokens_kernel<256, 1024>), grid, dim3(256), 0, stream, in, tokens, logprobs);
            HIP_TRY(hipGetLastError());
        }
        return (int)IVFPQ_OK;
    });
}
