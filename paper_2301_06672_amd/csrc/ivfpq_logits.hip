// Log-probabilities of tokens, the entropy and the best alternatives of rows of logits, mixed with listed tokens or not, the
// loss towards a teacher's listed tokens, and the gradients of all of these.
//
// Everything a row needs is a sum over exp2(t), t = (x - M) log2(e) / T with M the row's largest logit:
//   S = sum 2^t,  U = sum t 2^t,   log p_v = ln2 (t_v - log2 S),   entropy = ln2 (log2 S - U / S).
// t <= 0, so both terms of the entropy are non-negative.  Partial results (m, s, u) about a reference m combine by
// shifting: s 2^d, (u + d s) 2^d, d = (m - M) log2(e) / T.  A thread's reference may be up to 2^kSlack below its largest logit until its last
// shift; t is at most kSlack there, and the terms that cancel in u + d s are at most kSlack s each.  One pass over the logits is
// enough, and a row can be split between workgroups.  x - M is formed before the scale: a fused x scale - M scale would save one of eleven
// operations an element, but leaves fp32 where a row has nothing but masks of the type's lowest value.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ivfpq_float_key.hpp"
#include "ivfpq_hip_util.hpp"
#include "ivfpq_language_rules.hpp"
#include "ivfpq_values.hpp"

using namespace ivfpq;

namespace {

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / 64;
constexpr int kMostSplits = 64;                            // workgroups that share a row
// ... and where each leaves a list of its best keys, which have to be joined (131,072 bf16, 20 alternatives and 64 neighbours: one row in 8, 16,
// 32 parts 64, 36, 34 us, eight rows 64, 37, 41)
constexpr int kMostSplitsTop = 16;
constexpr int kMostTop = IVFPQ_MAX_MIXED;                  // keys a selection keeps
constexpr int kCandidates = 2048 - kMostTop;               // ... and takes in before it sorts
constexpr float kLeastPower = -150.f;                      // 2^t is 0 in fp32 below this: t is cut there before t 2^t

struct Partial { float m, s, u, unused; };

// ---- statistics

struct RowSum {
    float m = -INFINITY, s = 0.f, u = 0.f;
    RowSum() = default;
    __device__ explicit RowSum(const Partial& p) : m(p.m), s(p.s), u(p.u) {}
    // makes `most` the reference of the sums; most >= m
    __device__ inline void raise(float most, float scale) {
        const bool none = m == -INFINITY;
        const float d = none ? 0.f : (m - most) * scale;
        const float f = none ? 0.f : exp2_fast(d);
        u = __builtin_fmaf(fmaxf(d, kLeastPower), s, u) * f;
        s *= f;                                            // a NaN stays one
        m = most;
    }
    __device__ inline void join(RowSum b, float scale) {
        const float most = fmaxf(m, b.m);
        if (most == -INFINITY) {                           // nothing yet, or nothing but NaN
            s += b.s;
            u += b.u;
            return;
        }
        raise(most, scale);
        b.raise(most, scale);
        s += b.s;
        u += b.u;
    }
};

__device__ inline RowSum wave_join(RowSum a, float scale) {
    for (int off = 32; off; off >>= 1) {
        RowSum b;
        b.m = __shfl_xor(a.m, off);
        b.s = __shfl_xor(a.s, off);
        b.u = __shfl_xor(a.u, off);
        // the lower lane's part first in both, so that both get the same bits
        if (threadIdx.x & off) { const RowSum t = a; a = b; b = t; }
        a.join(b, scale);
    }
    return a;
}

// ---- the largest keys of a row

// A key orders logits descending and, among equal ones, tokens ascending; keys of a row are distinct.  0: none.
__device__ inline uint64_t token_key(float x, uint32_t token) {
    return ((uint64_t)ordered_key(x + 0.f) << 32) | (uint32_t)~token;      // -0 counts as +0
}
__device__ inline float key_value(uint64_t key) { return ordered_key_value((uint32_t)(key >> 32)); }
__device__ inline int key_token(uint64_t key) { return (int)~(uint32_t)key; }

struct Selection {
    alignas(16) uint64_t found[kCandidates + kMostTop];    // candidates, then room for the kept ones
    uint64_t kept[kMostTop];                   // the largest so far, descending
    uint64_t wave_bound[2][kRowWaves];
    int n_found;
};

// found[0, n) descending, n a power of two
__device__ inline void sort_found(Selection& sel, int n) {
    for (int len = 2; len <= n; len <<= 1)
        for (int step = len >> 1; step; step >>= 1) {
            for (int i = threadIdx.x; i < n / 2; i += kRowThreads) {
                const int a = 2 * i - (i & (step - 1)), b = a + step;
                const uint64_t x = sel.found[a], y = sel.found[b];
                if ((x < y) == ((a & len) == 0)) { sel.found[a] = y; sel.found[b] = x; }
            }
            __syncthreads();
        }
}

__device__ inline int power_of_two(int n) { return n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// The `want` largest of found[0, n) and kept[0, n_kept) become the kept ones; returns how many there are.  Few keys find their
// places by counting the larger ones, many are sorted.  Starts after a barrier and ends with one.
__device__ inline int keep_best(Selection& sel, int n, int n_kept, int want) {
    const int tid = threadIdx.x;
    for (int i = tid; i < n_kept; i += kRowThreads) sel.found[n + i] = sel.kept[i];
    const int total = n + n_kept;
    const int keep = total < want ? total : want;
    if (total <= 2 * kRowThreads) {
        // `share` neighbouring lanes count for one key; eight keys a lane are read at once, none (0) behind the last
        const int share = total <= 32 ? 8 : total <= 64 ? 4 : total <= 128 ? 2 : 1;
        const int padded = (total + 8 * share - 1) / (8 * share) * (8 * share);
        for (int i = total + tid; i < padded; i += kRowThreads) sel.found[i] = 0;
        __syncthreads();
        for (int i = tid / share; i < total; i += kRowThreads / share) {
            const uint64_t mine = sel.found[i];
            int place = 0;
            for (int j0 = tid % share * 2; j0 < padded; j0 += 8 * share) {
                uint64_t other[8];
#pragma unroll
                for (int o = 0; o < 8; o += 2) {
                    const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sel.found[j0 + o * share]);
                    other[o] = two.x;
                    other[o + 1] = two.y;
                }
#pragma unroll
                for (int o = 0; o < 8; ++o) place += other[o] > mine;
            }
            for (int off = 1; off < share; off <<= 1) place += __shfl_xor(place, off);
            if (place < want) sel.kept[place] = mine;      // the barrier above: kept has been copied
        }
    } else {
        const int padded = power_of_two(total);
        for (int i = total + tid; i < padded; i += kRowThreads) sel.found[i] = 0;
        __syncthreads();
        sort_found(sel, padded);
        for (int i = tid; i < keep; i += kRowThreads) sel.kept[i] = sel.found[i];
    }
    if (tid == 0) sel.n_found = 0;
    __syncthreads();
    return keep;
}

// Adds what `scan` finds to the kept keys.  scan(bound, push) calls push(key) for its keys >= bound, each at most once.  More than
// fit raise the bound to the want-th of those that did (keys below it cannot be among the best) and are looked for
// again; at least kCandidates - want keys are ruled out each time, so this ends.
// n_found is 0 on entry, and is on return; no wave is past the last barrier's reads.
template <class Scan>
__device__ inline int take_candidates(Selection& sel, uint64_t& bound, int n_kept, int want, Scan&& scan) {
    for (;;) {
        scan(bound, [&](uint64_t key) {
            const int at = atomicAdd(&sel.n_found, 1);     // the order of arrival does not matter: keys are sorted
            if (at < kCandidates) sel.found[at] = key;
        });
        __syncthreads();
        const int n = sel.n_found;
        __syncthreads();
        if (n == 0) return n_kept;
        if (n <= kCandidates) {
            n_kept = keep_best(sel, n, n_kept, want);
            if (n_kept == want && sel.kept[want - 1] > bound) bound = sel.kept[want - 1];
            return n_kept;
        }
        for (int i = kCandidates + threadIdx.x; i < 2048; i += kRowThreads) sel.found[i] = 0;
        if (threadIdx.x == 0) sel.n_found = 0;
        __syncthreads();
        sort_found(sel, 2048);
        if (sel.found[want - 1] > bound) bound = sel.found[want - 1];
        __syncthreads();
    }
}

// A lower bound of the want-th largest key of a workgroup, from one key of each lane (its largest, 0 if it has none).
// Either holds: with q = ceil(want / waves), every wave has q keys that are at least the smallest of the waves' q-th; and a
// wave has `want` keys that are at least its want-th.
__device__ inline uint64_t bound_of_best(Selection& sel, uint64_t mine, int want) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int larger = 0;
    for (int j = 0; j < 64; ++j) {
        const uint64_t other = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), j) << 32) |
                               (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, j);
        larger += other > mine;
    }
    if (lane == 0) sel.wave_bound[0][wave] = sel.wave_bound[1][wave] = 0;
    __builtin_amdgcn_wave_barrier();
    const int q = (want + kRowWaves - 1) / kRowWaves;
    if (larger == q - 1) sel.wave_bound[0][wave] = mine;         // lanes without a key share a place and a value, 0
    if (larger == want - 1) sel.wave_bound[1][wave] = mine;
    __syncthreads();
    uint64_t low = sel.wave_bound[0][0], high = sel.wave_bound[1][0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) {
        low = sel.wave_bound[0][w] < low ? sel.wave_bound[0][w] : low;
        high = sel.wave_bound[1][w] > high ? sel.wave_bound[1][w] : high;
    }
    __syncthreads();
    return low > high ? low : high;
}

// ---- what is done with a row's statistics

struct Listed {                       // tokens listed for every row, with a number each
    const int32_t* tokens;            // [n][k]
    const float* values;
    int k;
};

struct RowsIn {
    const void* data;
    long long stride;
    int vocab;
    float temperature, scale;         // scale = log2(e) / T
};

struct ScoreOut {
    const int32_t* targets;
    Listed near;
    float log_model, log_near;        // log(1 - weight), log(weight)
    int top, want;                    // want: keys to select, top plus the neighbours that may be among them
    float *logprobs, *entropy, *norms;
    int32_t* top_tokens;
    float* top_logprobs;
};

struct DistillOut {
    Listed teacher;
    float *loss, *norms;
};

struct MixShared {
    alignas(16) int token[IVFPQ_MAX_LISTED];
    float logp[IVFPQ_MAX_LISTED];     // of the mixture
    double sums[kRowWaves];
    float hit, model, near;           // the target's log-probability if it is listed; log weights in this row
};

// log(exp(a) + exp(b))
__device__ inline float log_add(float a, float b) {
    if (a != a || b != b) return a + b;
    const float most = fmaxf(a, b), least = fminf(a, b);
    if (most == -INFINITY) return most;
    return most + log1pf(expf(least - most));
}

__device__ inline void write_norms(float* norms, long long row, float m, float log_s, bool none) {
    if (!norms) return;
    norms[2 * row] = none ? -INFINITY : (log_s != log_s ? log_s : m);
    norms[2 * row + 1] = none ? -INFINITY : log_s;
}

// A row's target and its logit; read before the row, so that their latency is not at the end of it.
struct Target {
    int token = -1;                   // as given
    bool inside = false;
    float x = 0.f;
};
template <class T>
__device__ inline Target target_of(const RowsIn& in, const ScoreOut& out, long long row) {
    Target t;
    if (!out.targets) return t;
    t.token = out.targets[row];
    t.inside = t.token >= 0 && t.token < in.vocab;
    if (t.inside) t.x = (float)reinterpret_cast<const T*>(in.data)[row * in.stride + t.token];
    return t;
}
template <class T>
__device__ inline Target target_of(const RowsIn&, const DistillOut&, long long) { return Target{}; }

// All threads of a workgroup, on the statistics of one row; kept: its `n_kept` largest keys (TOP).
template <class T, bool TOP>
__device__ inline void finish_score(const RowsIn& in, const ScoreOut& out, long long row, const Target& target, RowSum sum, int n_kept, Selection* sel,
                                    MixShared& mix) {
    const int tid = threadIdx.x;
    const T* x = reinterpret_cast<const T*>(in.data) + row * in.stride;
    const bool none = sum.s == 0.f;                        // no logit above -inf (a largest one would have added 1)
    const float log_s = logf(sum.s);
    // log p of a logit
    auto model_logp = [&](float v) { return none ? -INFINITY : (v - sum.m) / in.temperature - log_s; };
    const float entropy = none ? 0.f : log_s - kLn2 * (sum.u / sum.s);
    const float unused = sum.s != sum.s ? sum.s : -INFINITY;       // in the place of an alternative: a row of NaN statistics has no other
    if (tid == 0) write_norms(out.norms, row, sum.m, log_s, none);

    if (out.near.k == 0) {
        if (tid == 0) {
            if (out.targets) out.logprobs[row] = target.inside ? model_logp(target.x) : 0.f;
            if (out.entropy) out.entropy[row] = entropy;
        }
        if constexpr (TOP)
            for (int i = tid; i < out.top; i += kRowThreads) {
                const float logp = i < n_kept ? model_logp(key_value(sel->kept[i])) : unused;
                const bool used = i < n_kept && logp != -INFINITY;       // a logit may be so far below the largest that this is no number of fp32
                out.top_tokens[row * out.top + i] = used ? key_token(sel->kept[i]) : -1;
                out.top_logprobs[row * out.top + i] = logp;
            }
        return;
    }

    // The mixture: m_v = (1 - w) p_v + w q_v differs from (1 - w) p_v at the listed tokens only, so its entropy is that of
    // the scaled model with the listed terms exchanged (summed in 64 bits: the exchange cancels).
    const int k = out.near.k;
    bool any = false;
    for (int j = tid; j < k; j += kRowThreads) {
        const int token = out.near.tokens[row * k + j];
        const bool used = token >= 0 && token < in.vocab;
        mix.token[j] = used ? token : -1;
        any |= used;
    }
    for (int j = k + tid; j < (k + 15) / 16 * 16; j += kRowThreads) mix.token[j] = -1;
    any = __syncthreads_or(any);
    const float log_model = none ? -INFINITY : any ? out.log_model : 0.f;
    const float log_near = !any ? -INFINITY : none ? 0.f : out.log_near;
    if (tid == 0) mix.hit = -INFINITY;
    double change = 0.0;                                   // of -sum m log m
    for (int j = tid; j < k; j += kRowThreads) {
        const int token = mix.token[j];
        if (token < 0) continue;
        const float model = log_model + model_logp((float)x[token]);
        const float mixed = log_add(model, log_near + out.near.values[row * k + j]);
        mix.logp[j] = mixed;
        if (model > kLeastPower || model != model) change += (double)expf(model) * (double)model;
        if (mixed > kLeastPower || mixed != mixed) change -= (double)expf(mixed) * (double)mixed;
    }
    change = block_sum<kRowThreads>(change, mix.sums);     // and a barrier behind mix.hit, mix.logp
    if (target.inside)
        for (int j = tid; j < k; j += kRowThreads)
            if (mix.token[j] == target.token) mix.hit = mix.logp[j];
    __syncthreads();
    if (tid == 0) {
        if (out.entropy) {
            const double base = none ? 0.0 : exp((double)log_model) * ((double)entropy - (double)log_model);
            const double h = base + change;
            out.entropy[row] = h > 0.0 || h != h ? (float)h : 0.f;
        }
        if (out.targets) {
            const bool listed = mix.hit > -INFINITY || mix.hit != mix.hit;
            out.logprobs[row] = !target.inside ? 0.f : listed ? mix.hit : log_model + model_logp(target.x);
        }
    }
    if constexpr (TOP) {
        // the kept tokens that are not listed, and the listed ones, by their mixed log-probabilities
        for (int i = tid; i < n_kept; i += kRowThreads) {
            const int token = key_token(sel->kept[i]);
            bool listed = false;
            for (int j = 0; j < k; j += 16) {              // -1 behind the last
                int4 some[4];
#pragma unroll
                for (int o = 0; o < 4; ++o) some[o] = *reinterpret_cast<const int4*>(&mix.token[j + 4 * o]);
#pragma unroll
                for (int o = 0; o < 4; ++o) listed |= some[o].x == token || some[o].y == token || some[o].z == token || some[o].w == token;
            }
            const float logp = log_model + model_logp(key_value(sel->kept[i]));
            if (!listed && logp > -INFINITY) sel->found[atomicAdd(&sel->n_found, 1)] = token_key(logp, (uint32_t)token);
        }
        for (int j = tid; j < k; j += kRowThreads)
            if (mix.token[j] >= 0 && mix.logp[j] > -INFINITY)
                sel->found[atomicAdd(&sel->n_found, 1)] = token_key(mix.logp[j], (uint32_t)mix.token[j]);
        __syncthreads();
        const int n = sel->n_found;
        if (tid < out.top) sel->kept[tid] = 0;             // a token listed twice, which a caller should not, leaves a place unused
        __syncthreads();
        const int best = keep_best(*sel, n, 0, out.top);
        for (int i = tid; i < out.top; i += kRowThreads) {
            const bool used = i < best && sel->kept[i];
            out.top_tokens[row * out.top + i] = used ? key_token(sel->kept[i]) : -1;
            out.top_logprobs[row * out.top + i] = used ? key_value(sel->kept[i]) : unused;
        }
    }
}

// The teacher's shares of its listed tokens: P_j of entry j = exp2((value_j - most) scale) / total, total 0 if no entry is used.
struct Teacher {
    float most, total;
};
__device__ inline bool teacher_uses(const Listed& l, long long row, int j, int vocab) {
    const int token = l.tokens[row * l.k + j];
    return token >= 0 && token < vocab && l.values[row * l.k + j] != -INFINITY;
}
template <int THREADS>
__device__ inline Teacher teacher_of(const Listed& l, long long row, int vocab, float scale, float* scratch) {
    float most = -INFINITY;
    for (int j = threadIdx.x; j < l.k; j += THREADS)
        if (teacher_uses(l, row, j, vocab)) most = fmaxf(most, l.values[row * l.k + j]);
    most = block_max<THREADS>(most, scratch);
    float total = 0.f;
    for (int j = threadIdx.x; j < l.k; j += THREADS)
        if (teacher_uses(l, row, j, vocab)) total += exp2_fast((l.values[row * l.k + j] - most) * scale);
    return Teacher{most, block_sum<THREADS>(total, scratch)};
}

// The row's loss, in every thread; x_of(j): the logit of entry j's token.
template <int THREADS, class XOf>
__device__ inline float loss_of(const RowsIn& in, const Listed& l, const Teacher& teacher, long long row, float m, float log_s, bool none, float* scratch, XOf&& x_of) {
    const float log_total = logf(teacher.total);
    float loss = 0.f;
    for (int j = threadIdx.x; j < l.k; j += THREADS) {
        if (!teacher_uses(l, row, j, in.vocab)) continue;
        const float at = (l.values[row * l.k + j] - teacher.most) * in.scale;
        const float share = exp2_fast(at) / teacher.total;
        if (share == 0.f) continue;
        const float logp = none ? -INFINITY : (x_of(j) - m) / in.temperature - log_s;
        loss += share * (__builtin_fmaf(at, kLn2, -log_total) - logp);
    }
    return block_sum<THREADS>(loss, scratch) * in.temperature * in.temperature;
}

template <class T>
__device__ inline void finish_distill(const RowsIn& in, const DistillOut& out, long long row, RowSum sum, float* scratch) {
    const T* x = reinterpret_cast<const T*>(in.data) + row * in.stride;
    const bool none = sum.s == 0.f;
    const float log_s = logf(sum.s);
    const Teacher teacher = teacher_of<kRowThreads>(out.teacher, row, in.vocab, in.scale, scratch);
    const float loss = loss_of<kRowThreads>(in, out.teacher, teacher, row, sum.m, log_s, none, scratch,
                                            [&](int j) { return (float)x[out.teacher.tokens[row * out.teacher.k + j]]; });
    if (threadIdx.x == 0) {
        out.loss[row] = loss;
        write_norms(out.norms, row, sum.m, log_s, none);
    }
}

// ---- the pass over the logits

// 16-byte chunks that a thread holds at once
constexpr int kRowChunks = 2;

// Whole chunks c0, c0 + kRowThreads, ... of a row for a thread's place; from `end` on the last one again.  No branch, so that the
// loads of the next tile stay in flight while this one is added up.
template <class T>
__device__ inline void load_tile(const RowChunks<T>& row, int c0, int end, Chunk<T> (&k)[kRowChunks]) {
#pragma unroll
    for (int i = 0; i < kRowChunks; ++i) k[i].bits = row.base[(uint32_t)min(c0 + i * kRowThreads + (int)threadIdx.x, end - 1)];
}

template <class T>
__device__ inline void clear(Chunk<T>& k) {
    float none[Chunk<T>::VEC];
#pragma unroll
    for (int j = 0; j < Chunk<T>::VEC; ++j) none[j] = -INFINITY;
    k.narrow(none);
}

// -inf in the place of what load_tile read again
template <class T>
__device__ inline void cut_tile(int c0, int end, Chunk<T> (&k)[kRowChunks]) {
    if (c0 + kRowChunks * kRowThreads <= end) return;
#pragma unroll
    for (int i = 0; i < kRowChunks; ++i)
        if (c0 + i * kRowThreads + (int)threadIdx.x >= end) clear(k[i]);
}

// The row's values before its first whole chunk (`front`) and behind its last one (`back`), a chunk in each of the first two
// threads; -inf elsewhere.  Returns the chunk that it is, for its tokens.
template <class T>
__device__ inline int load_edges(const RowChunks<T>& row, bool front, bool back, Chunk<T> (&k)[1]) {
    clear(k[0]);
    const int c = threadIdx.x == 0 ? 0 : row.end_whole();
    if ((threadIdx.x == 0 && front) || (threadIdx.x == 1 && back)) k[0] = row.load(c);
    return c;
}

template <class T, int N>
__device__ inline void largest_of_chunks(const Chunk<T> (&k)[N], float (&most)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float x[Chunk<T>::VEC];
        k[i].widen(x);
        most[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < Chunk<T>::VEC; j += 2) most[i] = max3(most[i], x[j], x[j + 1]);
    }
}

// Adds the chunks to a thread's sums; leaves the maximum of every chunk, and of all so far in `largest`.  The reference follows the
// maximum only when that is over 2^kSlack of it: most tiles raise some lane's maximum by a little, and a raise costs as
// much as an element.  The sums' parts stay within 2^kSlack of their place, so nothing is lost.  A tile's values are added up among
// themselves first: one after the other onto a sum near its end, small ones are rounded away (65,536 normal logits, in log S: 3.5e-7 too
// little on average against 0.6e-7).
constexpr float kSlack = 4.f;
template <class T, bool ENTROPY, int N>
__device__ inline void add_tile(Chunk<T> (&k)[N], float scale, RowSum& sum, float& largest, float (&most)[N]) {
    constexpr int VEC = Chunk<T>::VEC;
    float x[N][VEC];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        k[i].widen(x[i]);
        most[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < VEC; j += 2) most[i] = max3(most[i], x[i][j], x[i][j + 1]);
        largest = fmaxf(largest, most[i]);
    }
    if ((largest - sum.m) * scale > kSlack) sum.raise(largest, scale);
    const float ref = sum.m == -INFINITY ? 0.f : sum.m;     // nothing but -inf so far: t = -inf, not a NaN
    float s[N], u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float e[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float t = (x[i][j] - ref) * scale;
            e[j] = exp2_fast(t);
            if constexpr (ENTROPY) u[i] = j ? __builtin_fmaf(fmaxf(t, kLeastPower), e[j], u[i]) : fmaxf(t, kLeastPower) * e[j];
        }
        s[i] = tree_sum<VEC>(e);
    }
    sum.s += tree_sum<N>(s);
    if constexpr (ENTROPY) sum.u += tree_sum<N>(u);
}

// The largest key of a thread's chunks, 0 if they hold nothing above -inf.
template <class T, int N>
__device__ inline uint64_t best_of_tile(Chunk<T> (&k)[N], const float (&most)[N], int first) {
    constexpr int VEC = Chunk<T>::VEC;
    float top = most[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, most[i]);
    int at = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
        float x[VEC];
        k[i].forget_widened();
        k[i].widen(x);
#pragma unroll
        for (int j = VEC - 1; j >= 0; --j) at = x[j] == top ? i * kRowThreads * VEC + j : at;
    }
    return top > -INFINITY ? token_key(top, (uint32_t)(first + at)) : 0;
}

enum class RowMode { kScore, kScoreTop, kDistill };

struct RowShared {
    Partial waves[kRowWaves];
    float scratch[kRowWaves];
};
template <RowMode MODE> struct RowLds { RowShared rows; MixShared mix; };
template <> struct RowLds<RowMode::kScoreTop> { RowShared rows; Selection sel; };
template <> struct RowLds<RowMode::kDistill> { RowShared rows; };

// Where a mixture's numbers are: with a selection in the back of its candidates, of which the last merge uses 2 kMostTop and
// what fills up a step of counting.
template <RowMode MODE>
__device__ inline MixShared& mix_of(RowLds<MODE>& lds) {
    if constexpr (MODE == RowMode::kScoreTop) {
        constexpr int kFront = 3 * kMostTop;
        static_assert(sizeof(MixShared) <= sizeof(lds.sel.found) - kFront * sizeof(uint64_t), "room for both");
        return *reinterpret_cast<MixShared*>(lds.sel.found + kFront);
    } else {
        return lds.mix;
    }
}

struct RowSplit {
    int splits, chunks;               // workgroups a row, chunks of each
    Partial* partials;                // [n][splits]; null with one workgroup a row
    uint64_t* keys;                   // [n][splits][want], descending, 0 where there are fewer
};

// the statistics of the workgroup's threads, in all of them
__device__ inline RowSum block_join(RowSum sum, float scale, RowShared& lds) {
    sum = wave_join(sum, scale);
    if ((threadIdx.x & 63) == 0) lds.waves[threadIdx.x >> 6] = Partial{sum.m, sum.s, sum.u, 0.f};
    __syncthreads();
    sum = RowSum(lds.waves[0]);
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) sum.join(RowSum(lds.waves[w]), scale);
    return sum;
}

template <class T, RowMode MODE, class Out>
__device__ inline void finish_row(const RowsIn& in, const Out& out, long long row, const Target& target, RowSum sum, int n_kept, RowLds<MODE>& lds) {
    if constexpr (MODE == RowMode::kScoreTop) finish_score<T, true>(in, out, row, target, sum, n_kept, &lds.sel, mix_of<MODE>(lds));
    else if constexpr (MODE == RowMode::kScore) finish_score<T, false>(in, out, row, target, sum, 0, nullptr, mix_of<MODE>(lds));
    else finish_distill<T>(in, out, row, sum, lds.rows.scratch);
}

// The keys of a tile that are at least b, b = 0 for all but -inf
template <class T, int N, class Push>
__device__ inline void scan_tile(Chunk<T> (&k)[N], const float (&most)[N], int first, uint64_t b, Push&& push) {
    constexpr int VEC = Chunk<T>::VEC;
    const float least = b ? key_value(b) : -INFINITY;
    asm volatile("" : "+v"(first));                        // tokens are formed where they are needed, not kept in registers
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!(most[i] >= least)) continue;
        float x[VEC];
        k[i].forget_widened();
        k[i].widen(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (x[j] >= least && x[j] > -INFINITY) {
                const uint64_t key = token_key(x[j], (uint32_t)(first + i * kRowThreads * VEC + j));
                if (key >= b) push(key);
            }
    }
}

// The best keys of chunks [begin, end), whole or not, for rows where too many keys passed the bounds of the one pass: a chunk a
// thread at a time, each time bounded by the best of these while too few keys are kept.
template <class T>
__device__ inline int select_step_by_step(const RowChunks<T>& row, int begin, int end, int want, Selection& sel) {
    uint64_t bound = 0;
    int n_kept = 0;
    for (int c0 = begin; c0 < end; c0 += kRowThreads) {
        const int c = c0 + (int)threadIdx.x, first = c * Chunk<T>::VEC - row.lead;
        Chunk<T> k[1];
        float most[1];
        if (c < end) k[0] = row.load(c);
        else clear(k[0]);
        largest_of_chunks(k, most);
        if (n_kept < want) bound = bound_of_best(sel, best_of_tile(k, most, first), want);
        n_kept = take_candidates(sel, bound, n_kept, want, [&](uint64_t b, auto push) { scan_tile(k, most, first, b, push); });
    }
    return n_kept;
}

// One workgroup: the whole chunks [split * chunks, ...) of a row; the row's first workgroup takes what lies before them too, and
// its last one what lies behind.
//
// Alternatives: the first tile's keys above a bound from its lanes' best are merged at once, and what passes the want-th of
// those is collected from the next tiles without a barrier, merged after 4, 16, ... tiles (a bound from N tiles lets about as
// many of the next N pass as are wanted).
//
// Measured on bf16, calls in a row, inputs of over 1 GB in turn: 4,096 x 65,536 without entropy 99 us (5.4 TB/s), with entropy 101, with
// 20 alternatives too 135 (4.0 TB/s: normal logits in any order; 115 where the likely tokens are the low ones, whose bounds let fewer pass);
// 2,048 rows with entropy 55 us (4.9 TB/s), 80 right after a kernel that wrote as much.  Reading bounds the first; the others are near what
// the vector ALU takes, about ten instructions and an exponential (of two) a logit.  Tiles of two chunks a thread: of four, alternatives
// take 1.5 times as long (registers: five workgroups a CU for six, and more to look through).
template <class T, RowMode MODE, class Out>
__global__ __launch_bounds__(kRowThreads, 6) void row_statistics_kernel(RowsIn in, RowSplit split, Out out) {
    constexpr int VEC = Chunk<T>::VEC;
    constexpr bool TOP = MODE == RowMode::kScoreTop, ENTROPY = MODE != RowMode::kDistill;
    __shared__ RowLds<MODE> lds;
    const long long r = blockIdx.x / (unsigned)split.splits;
    const int part = blockIdx.x % (unsigned)split.splits;
    const RowChunks<T> row(in.data, r, in.stride, in.vocab);
    const int begin = row.first_whole() + part * split.chunks;
    const int end = min(begin + split.chunks, row.end_whole());
    const bool last = part + 1 == split.splits;
    const Target target = split.splits == 1 ? target_of<T>(in, out, r) : Target{};
    const bool front = part == 0 && !row.whole(0), back = last && row.end_whole() > 0 && row.end % VEC;
    RowSum sum;
    float largest = -INFINITY;
    uint64_t bound = 0;
    int n_kept = 0, want = 0, tiles = 0, merge_at = 1;
    bool many = false;                                     // more candidates than there is room for
    auto collect = [&](uint64_t key) {
        if constexpr (TOP) {
            const int at = atomicAdd(&lds.sel.n_found, 1);         // the order of arrival does not matter: keys are sorted
            if (at < kCandidates) lds.sel.found[at] = key;
        }
    };
    auto merge = [&] {
        if constexpr (TOP) {
            __syncthreads();
            const int n = lds.sel.n_found;
            __syncthreads();
            many = n > kCandidates;
            if (n > 0 && !many) n_kept = keep_best(lds.sel, n, n_kept, want);
            if (n_kept == want) bound = lds.sel.kept[want - 1];
        }
    };
    if constexpr (TOP) {
        want = out.want;
        if (threadIdx.x == 0) lds.sel.n_found = 0;
        __syncthreads();
    }
    Chunk<T> now[kRowChunks], next[kRowChunks], edge[1];
    int edge_token = 0;
    if (front || back) edge_token = load_edges(row, front, back, edge) * VEC - row.lead;       // ahead, as the tiles are
    if (begin < end) load_tile(row, begin, end, now);
    for (int c0 = begin; c0 < end; c0 += kRowChunks * kRowThreads) {
        const int c1 = c0 + kRowChunks * kRowThreads;
        load_tile(row, c1, end, next);
        cut_tile(c0, end, now);
        float most[kRowChunks];
        add_tile<T, ENTROPY>(now, in.scale, sum, largest, most);
        if constexpr (TOP) {
            const int first = (c0 + (int)threadIdx.x) * VEC - row.lead;
            if (c0 == begin) bound = bound_of_best(lds.sel, best_of_tile(now, most, first), want);
            if (!many) {
                scan_tile(now, most, first, bound, collect);
                if (++tiles == merge_at) {
                    merge_at *= 4;
                    merge();
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kRowChunks; ++i) now[i] = next[i];
    }
    if (front || back) {
        float most[1];
        add_tile<T, ENTROPY>(edge, in.scale, sum, largest, most);
        if (TOP && !many) scan_tile(edge, most, edge_token, bound, collect);
    }
    if constexpr (TOP) {
        if (!many) merge();
        if (many) {
            __syncthreads();
            if (threadIdx.x == 0) lds.sel.n_found = 0;
            __syncthreads();
            n_kept = select_step_by_step(row, part == 0 ? 0 : min(begin, end), last ? row.count() : end, want, lds.sel);
        }
    }
    if (largest > sum.m) sum.raise(largest, in.scale);
    sum = block_join(sum, in.scale, lds.rows);
    if (split.splits == 1) {
        __syncthreads();
        finish_row<T, MODE>(in, out, r, target, sum, n_kept, lds);
        return;
    }
    const long long at = r * split.splits + part;
    if (threadIdx.x == 0) split.partials[at] = Partial{sum.m, sum.s, sum.u, 0.f};
    if constexpr (TOP)
        for (int i = threadIdx.x; i < want; i += kRowThreads) split.keys[at * want + i] = i < n_kept ? lds.sel.kept[i] : 0;
}

// One workgroup a row: joins what the row's workgroups left.  A chain of latencies: one row of 131,072 with 20 alternatives mixed with
// 64 neighbours 16 us beside the 18 us of its statistics.
template <class T, RowMode MODE, class Out>
__global__ __launch_bounds__(kRowThreads) void row_join_kernel(RowsIn in, RowSplit split, Out out) {
    __shared__ RowLds<MODE> lds;
    const long long r = blockIdx.x;
    const Target target = target_of<T>(in, out, r);
    RowSum sum;
    if ((int)threadIdx.x < split.splits) sum = RowSum(split.partials[r * split.splits + threadIdx.x]);
    sum = block_join(sum, in.scale, lds.rows);
    int n_kept = 0;
    if constexpr (MODE == RowMode::kScoreTop) {
        const int want = out.want;
        const uint64_t* keys = split.keys + r * split.splits * (long long)want;
        // every workgroup's q-th largest key bounds q keys from below; together splits * q >= want
        const int q = (want + split.splits - 1) / split.splits;
        static_assert(kMostSplits <= 64, "one wave reads them all");
        uint64_t low = ~(uint64_t)0, high = 0;
        const int p = threadIdx.x & 63;
        if (p < split.splits) {
            low = keys[(long long)p * want + q - 1];
            high = keys[(long long)p * want + want - 1];
        }
        for (int off = 32; off; off >>= 1) {
            const uint64_t a = __shfl_xor((unsigned long long)low, off), b = __shfl_xor((unsigned long long)high, off);
            low = a < low ? a : low;
            high = b > high ? b : high;
        }
        uint64_t bound = low > high ? low : high;
        if (threadIdx.x == 0) lds.sel.n_found = 0;
        __syncthreads();
        n_kept = take_candidates(lds.sel, bound, 0, want, [&](uint64_t b, auto push) {
            constexpr int kAhead = 8;                      // loads in flight: this kernel is little more than their latency
            const int n = split.splits * want;
            for (int i = threadIdx.x; i < n; i += kAhead * kRowThreads) {
                uint64_t some[kAhead];
#pragma unroll
                for (int o = 0; o < kAhead; ++o) some[o] = i + o * kRowThreads < n ? keys[i + o * kRowThreads] : 0;
#pragma unroll
                for (int o = 0; o < kAhead; ++o)
                    if (some[o] >= b && some[o]) push(some[o]);
            }
        });
    }
    __syncthreads();
    finish_row<T, MODE>(in, out, r, target, sum, n_kept, lds);
}

// ---- gradients

struct GradIn {
    const float* norms;               // [n][2]
    void* grad;
    long long grad_stride;
    int chunks;                       // of a workgroup
    int splits;
};
struct PolicyGrad {
    const int32_t* targets;
    const float *entropy, *by_logprob, *by_entropy;
};
struct DistillGrad {
    Listed teacher;
    const float* row_grads;
};

template <int THREADS>
struct GradShared {
    float scratch[THREADS / 64];
    alignas(16) int token[IVFPQ_MAX_LISTED];
    float share[IVFPQ_MAX_LISTED];
    float x[IVFPQ_MAX_LISTED];
};

// The listed tokens in [token0, token1) with their logits and what they add to the gradient, -w P_j; -1 for unused entries and up
// to a multiple of 16 behind them.  Before anything is written: the gradient may lie over the logits.
template <class T, int THREADS>
__device__ inline void stage_listed(const Listed& l, const RowChunks<T>& row, long long r, int vocab, const Teacher& teacher, float scale, float w, int token0,
                                    int token1, GradShared<THREADS>& lds) {
    for (int j = threadIdx.x; j < (l.k + 15) / 16 * 16; j += THREADS) {
        const bool used = j < l.k && teacher_uses(l, r, j, vocab);
        const int token = used ? l.tokens[r * l.k + j] : -1;
        lds.token[j] = token;
        if (!used) continue;
        lds.share[j] = -w * exp2_fast((l.values[r * l.k + j] - teacher.most) * scale) / teacher.total;
        lds.x[j] = token >= token0 && token < token1 ? row.value(token) : 0.f;
    }
}

// The elements of the listed tokens, once more and whole, behind a barrier after the others.  Entries of one token add up, in
// their order, at the first of them.
template <class T, int THREADS, class Dense>
__device__ inline void write_listed(int k, int token0, int token1, const GradShared<THREADS>& lds, T* grad, Dense&& dense) {
    for (int j = threadIdx.x; j < k; j += THREADS) {
        const int token = lds.token[j];
        if (token < token0 || token >= token1) continue;
        int same = 0;
        for (int i = 0; i < k; i += 16) {
            int4 some[4];
#pragma unroll
            for (int o = 0; o < 4; ++o) some[o] = *reinterpret_cast<const int4*>(&lds.token[i + 4 * o]);
#pragma unroll
            for (int o = 0; o < 4; ++o) same += (some[o].x == token) + (some[o].y == token) + (some[o].z == token) + (some[o].w == token);
        }
        float share = lds.share[j];
        bool first = true;
        if (same > 1)
            for (int i = 0; i < k; ++i)
                if (i != j && lds.token[i] == token) {
                    first &= i > j;
                    share += lds.share[i];
                }
        if (first) grad[token] = (T)(dense(lds.x[j]) + share);
    }
}

// grad_v = p_v (a + b t_v), t_v = log2 p_v, plus a term at a few listed tokens; a row without a distribution has zeros.
// One workgroup: the chunks [split * chunks, ...) of a row.  The listed tokens' logits are read before anything is
// written (the gradient may lie over the logits) and their elements written again after a barrier.  Bound by memory: 2,048 x 65,536 bf16
// 106 us, 5.1 TB/s of reads and writes; 86 right after the statistics, with part of the logits still in the last-level cache.
template <class T, bool BY_ENTROPY, class How>
__global__ __launch_bounds__(kRowThreads) void row_gradient_kernel(RowsIn in, GradIn g, How how) {
    constexpr int VEC = Chunk<T>::VEC;
    constexpr bool POLICY = std::is_same<How, PolicyGrad>::value;
    __shared__ GradShared<kRowThreads> lds;
    const int tid = threadIdx.x;
    const long long r = blockIdx.x / (unsigned)g.splits;
    const int part = blockIdx.x % (unsigned)g.splits;
    const RowChunks<T> row(in.data, r, in.stride, in.vocab), to(g.grad, r, g.grad_stride, in.vocab);
    T* grad = const_cast<T*>(to.row);
    const int begin = part * g.chunks;
    const int end = min(begin + g.chunks, row.count());
    const int token0 = max(begin * VEC - row.lead, 0), token1 = min(end * VEC - row.lead, in.vocab);    // the workgroup's
    const float m = g.norms[2 * r], log2_s = g.norms[2 * r + 1] * kLog2E;
    const bool none = m == -INFINITY;
    float a = 0.f, b = 0.f;
    int k = 0;
    if constexpr (POLICY) {
        const float by_logprob = how.by_logprob ? how.by_logprob[r] : 0.f;
        const int target = how.targets ? how.targets[r] : -1;
        const bool wanted = target >= 0 && target < in.vocab;
        const float gl = wanted ? by_logprob / in.temperature : 0.f;
        a = -gl;
        if constexpr (BY_ENTROPY) {
            const float gh = how.by_entropy[r] / in.temperature;
            a -= gh * how.entropy[r];
            b = -gh * kLn2;
        }
        k = wanted && how.by_logprob ? 1 : 0;
        if (tid > 0 && tid < 16) lds.token[tid] = -1;
        if (tid == 0 && k) {
            lds.token[0] = target;
            lds.share[0] = gl;
            lds.x[0] = target >= token0 && target < token1 ? row.value(target) : 0.f;
        }
    } else {
        const Teacher teacher = teacher_of<kRowThreads>(how.teacher, r, in.vocab, in.scale, lds.scratch);
        const float w = in.temperature * (how.row_grads ? how.row_grads[r] : 1.f);
        k = how.teacher.k;
        stage_listed(how.teacher, row, r, in.vocab, teacher, in.scale, w, token0, token1, lds);
        a = teacher.total == 0.f ? 0.f : w;                // a NaN among the values stays one
    }
    __syncthreads();
    auto dense = [&](float x) {
        const float t = __builtin_fmaf(x - m, in.scale, -log2_s);
        const float p = exp2_fast(t);
        if constexpr (BY_ENTROPY) return p * __builtin_fmaf(b, fmaxf(t, kLeastPower), a);
        else return p * a;
    };
    const bool alike = to.lead == row.lead;                // chunks of both lie alike
    for (int c = begin + tid; c < end; c += kRowThreads) {
        float x[VEC];
        row.load(c).widen(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = none ? 0.f : dense(x[j]);
        if (alike && row.whole(c)) {
            Chunk<T> y;
            y.narrow(x);
            const_cast<uint4*>(to.base)[c] = y.bits;
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int v = c * VEC + j - row.lead;
                if (v >= 0 && v < in.vocab) grad[v] = (T)x[j];
            }
        }
    }
    if (none) return;
    __syncthreads();
    write_listed(k, token0, token1, lds, grad, dense);
}

// Loss and gradient in one pass, for rows that fit the registers of a workgroup (HELD 16-byte chunks a thread): every
// logit is read once and every element of the gradient written once.  4,096 x 65,536 bf16 (512 threads): 260 us, 4.1 TB/s (a copy: 4.65); two
// workgroups a CU, so that one row's loads run beside the other's exponentials and stores.  Of 1,024 threads a CU holds one.
template <class T, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void distill_step_kernel(RowsIn in, DistillGrad how, float* __restrict__ loss, void* grads, long long grad_stride) {
    constexpr int VEC = Chunk<T>::VEC;
    __shared__ GradShared<THREADS> lds;
    const int tid = threadIdx.x;
    const long long r = blockIdx.x;
    const RowChunks<T> row(in.data, r, in.stride, in.vocab), to(grads, r, grad_stride, in.vocab);
    T* grad = const_cast<T*>(to.row);
    const int begin = row.first_whole(), end = row.end_whole();
    const bool front = !row.whole(0), back = end > 0 && row.end % VEC;
    const bool alike = to.lead == row.lead;                // chunks of both lie alike
    Chunk<T> held[HELD], edge[1];
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (begin + i * THREADS < end) held[i].bits = row.base[min(begin + i * THREADS + tid, end - 1)];
    const int edge_chunk = load_edges(row, front, back, edge);
    const Teacher teacher = teacher_of<THREADS>(how.teacher, r, in.vocab, in.scale, lds.scratch);
    const float w = in.temperature * (how.row_grads ? how.row_grads[r] : 1.f);
    stage_listed(how.teacher, row, r, in.vocab, teacher, in.scale, w, 0, in.vocab, lds);

    float most[1];
    largest_of_chunks(edge, most);
    float m = most[0];
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (begin + i * THREADS < end) {                   // a chunk that stands in for one behind the last changes no maximum
            float x[VEC];
            held[i].widen(x);
#pragma unroll
            for (int j = 0; j < VEC; j += 2) m = max3(m, x[j], x[j + 1]);
        }
    m = block_max<THREADS>(m, lds.scratch);                // and a barrier behind stage_listed
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
    auto add = [&](Chunk<T>& k) {
        float x[VEC];
        k.forget_widened();
        k.widen(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = exp2_fast((x[j] - ref) * in.scale);
        s += tree_sum<VEC>(x);
    };
    if (front || back) add(edge[0]);
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (begin + i * THREADS + tid < end) add(held[i]);
    s = block_sum<THREADS>(s, lds.scratch);
    const bool none = s == 0.f;
    const float log_s = logf(s), log2_s = log_s * kLog2E;
    if (s != s) m = s;                                     // a NaN that is no number's equal is no maximum either
    const float a = teacher.total == 0.f ? 0.f : w;
    auto dense = [&](float x) { return a * exp2_fast(__builtin_fmaf(x - m, in.scale, -log2_s)); };
    const float row_loss = loss_of<THREADS>(in, how.teacher, teacher, r, m, log_s, none, lds.scratch, [&](int j) { return lds.x[j]; });
    if (tid == 0) loss[r] = row_loss;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (begin + i * THREADS + tid < end) {
            float x[VEC];
            held[i].forget_widened();
            held[i].widen(x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = none ? 0.f : dense(x[j]);
            const int c = begin + i * THREADS + tid;
            if (alike) {
                Chunk<T> y;
                y.narrow(x);
                const_cast<uint4*>(to.base)[c] = y.bits;
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) grad[c * VEC + j - row.lead] = (T)x[j];
            }
        }
    if ((tid == 0 && front) || (tid == 1 && back)) {
        float x[VEC];
        edge[0].widen(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int v = edge_chunk * VEC + j - row.lead;
            if (v >= 0 && v < in.vocab) grad[v] = (T)(none ? 0.f : dense(x[j]));
        }
    }
    if (none) return;
    __syncthreads();
    write_listed(how.teacher.k, 0, in.vocab, lds, grad, dense);
}

// ---- launches

constexpr int64_t kMostRows = 1 << 21;                      // a launch has fewer than 2^32 threads
constexpr float kLeastTemperature = 1e-6f, kMostTemperature = 1e6f;       // T^2 and log2(e) / T stay moderate

// How a row is dealt to workgroups: as many as run at once (six on each of 256 CUs; a few more would take as long as that many
// again), at least a chunk for every thread, at most most_splits.
RowSplit split_rows(int64_t n, int32_t vocab, int vec, int most_splits) {
    constexpr int64_t kAtOnce = 6 * 256;
    const int64_t chunks = ((int64_t)vocab + vec - 1) / vec + 1;      // of a row at the worst alignment
    const int64_t useful = (chunks + kRowThreads - 1) / kRowThreads;
    const int64_t splits = std::min<int64_t>({std::max<int64_t>(kAtOnce / n, 1), useful, most_splits});
    RowSplit s{};
    s.chunks = (int)((chunks + splits - 1) / splits);
    s.chunks = (s.chunks + kRowThreads - 1) / kRowThreads * kRowThreads;
    s.splits = (int)((chunks + s.chunks - 1) / s.chunks);
    return s;
}

int check_rows(const char* what, const void* data, int32_t dtype, int64_t n, int32_t vocab, int64_t stride, float temperature) {
    if (!known_dtype(dtype)) return fail(IVFPQ_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (n < 0 || vocab < 1) return fail(IVFPQ_EINVAL, "%s: bad shape (n=%lld vocab=%d)", what, (long long)n, vocab);
    if (vocab > (1 << 30)) return fail(IVFPQ_EUNSUPPORTED, "%s: vocab=%d (limit 2^30)", what, vocab);
    if (n > kMostRows) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld (limit 2^21 rows per call)", what, (long long)n);
    if (n > 1 && stride < vocab) return fail(IVFPQ_EINVAL, "%s: row stride %lld below vocab=%d", what, (long long)stride, vocab);
    if (!(temperature >= kLeastTemperature && temperature <= kMostTemperature))
        return fail(IVFPQ_EINVAL, "%s: temperature outside [%g, %g]", what, (double)kLeastTemperature, (double)kMostTemperature);
    if (n > 0 && !data) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)data % value_bytes(dtype)) return fail(IVFPQ_EINVAL, "%s: logits are not aligned to their type", what);
    return IVFPQ_OK;
}

int check_grad(const char* what, const void* logits, int64_t stride, const void* grad, int32_t dtype, int64_t n, int32_t vocab, int64_t grad_stride) {
    if (n > 0 && !grad) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    if (n > 1 && grad_stride < vocab) return fail(IVFPQ_EINVAL, "%s: gradient stride %lld below vocab=%d", what, (long long)grad_stride, vocab);
    if ((uintptr_t)grad % value_bytes(dtype)) return fail(IVFPQ_EINVAL, "%s: the gradient is not aligned to its type", what);
    if (n > 0) {
        const size_t vb = value_bytes(dtype);
        const uintptr_t a = (uintptr_t)logits, b = (uintptr_t)grad;
        const uintptr_t a1 = a + ((size_t)(n - 1) * stride + vocab) * vb, b1 = b + ((size_t)(n - 1) * grad_stride + vocab) * vb;
        const size_t width = (size_t)vocab * vb, pitch = (size_t)stride * vb;
        const size_t apart = n > 1 ? (a < b ? b - a : a - b) % pitch : 0;         // columns of one wider matrix
        const bool beside = n > 1 && stride == grad_stride && apart >= width && apart <= pitch - width;
        if (a < b1 && b < a1 && !beside && !(a == b && (n == 1 || stride == grad_stride)))
            return fail(IVFPQ_EINVAL, "%s: the gradient overlaps the logits without lying over them", what);
    }
    return IVFPQ_OK;
}

int check_listed(const char* what, const int32_t* tokens, const float* values, int64_t n, int32_t k) {
    if (k < 1 || k > IVFPQ_MAX_LISTED) return fail(IVFPQ_EINVAL, "%s: k=%d outside [1, %d]", what, k, (int)IVFPQ_MAX_LISTED);
    if (n > 0 && (!tokens || !values)) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    return IVFPQ_OK;
}

int check_workspace(const char* what, const void* ws, size_t bytes, size_t need) {
    if (need == 0) return IVFPQ_OK;
    if (!ws) return fail(IVFPQ_EINVAL, "%s: null workspace", what);
    if ((uintptr_t)ws % kAlign) return fail(IVFPQ_EINVAL, "%s: workspace not aligned to %zu bytes", what, kAlign);
    if (bytes < need) return fail(IVFPQ_ENOSPACE, "%s: workspace %zu bytes, need %zu", what, bytes, need);
    return IVFPQ_OK;
}

RowsIn rows_in(const void* data, int64_t stride, int32_t vocab, float temperature) {
    return RowsIn{data, stride, vocab, temperature, (float)(1.4426950408889634 / (double)temperature)};
}

// scratch of the split rows of `n`: partial sums, then keys
size_t split_bytes(int64_t n, const RowSplit& s, int want) {
    if (s.splits == 1) return 0;
    return align_up((size_t)n * s.splits * sizeof(Partial)) + align_up((size_t)n * s.splits * want * sizeof(uint64_t));
}

// the largest over the value types
size_t row_workspace(int64_t n, int32_t vocab, int want) {
    const int most = want ? kMostSplitsTop : kMostSplits;
    if (n < 1 || vocab < 1 || vocab > (1 << 30) || n > kMostRows) return 0;
    return std::max(split_bytes(n, split_rows(n, vocab, 4, most), want), split_bytes(n, split_rows(n, vocab, 8, most), want));
}

template <class T, RowMode MODE, class Out>
int launch_rows(int64_t n, const RowsIn& in, const Out& out, void* ws, hipStream_t stream) {
    RowSplit s = split_rows(n, in.vocab, Chunk<T>::VEC, MODE == RowMode::kScoreTop ? kMostSplitsTop : kMostSplits);
    if (s.splits > 1) {
        s.partials = (Partial*)ws;
        s.keys = (uint64_t*)((char*)ws + align_up((size_t)n * s.splits * sizeof(Partial)));
    }
    hipLaunchKernelGGL((row_statistics_kernel<T, MODE, Out>), dim3((unsigned)(n * s.splits)), dim3(kRowThreads), 0, stream, in, s, out);
    HIP_TRY(hipGetLastError());
    if (s.splits > 1) {
        hipLaunchKernelGGL((row_join_kernel<T, MODE, Out>), dim3((unsigned)n), dim3(kRowThreads), 0, stream, in, s, out);
        HIP_TRY(hipGetLastError());
    }
    return IVFPQ_OK;
}

template <class T, bool BY_ENTROPY, class How>
int launch_gradient(int64_t n, const RowsIn& in, GradIn g, const How& how, hipStream_t stream) {
    const RowSplit s = split_rows(n, in.vocab, Chunk<T>::VEC, kMostSplits);
    g.splits = s.splits;
    g.chunks = s.chunks;
    hipLaunchKernelGGL((row_gradient_kernel<T, BY_ENTROPY, How>), dim3((unsigned)(n * s.splits)), dim3(kRowThreads), 0, stream, in, g, how);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

int token_logprobs(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride, const int32_t* d_targets,
                   float temperature, int32_t top, const int32_t* d_neighbour_tokens, const float* d_neighbour_logprobs,
                   int32_t n_neighbours, float weight, float* d_logprobs, float* d_entropy, float* d_norms, int32_t* d_top_tokens,
                   float* d_top_logprobs, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    const char* what = "ivfpq_token_logprobs";
    if (int s = check_rows(what, d_logits, dtype, n, vocab, row_stride, temperature)) return s;
    if (top < 0 || top > IVFPQ_MAX_TOP) return fail(IVFPQ_EINVAL, "%s: top=%d outside [0, %d]", what, top, (int)IVFPQ_MAX_TOP);
    if (n_neighbours < 0 || n_neighbours > IVFPQ_MAX_LISTED)
        return fail(IVFPQ_EINVAL, "%s: n_neighbours=%d outside [0, %d]", what, n_neighbours, (int)IVFPQ_MAX_LISTED);
    if (top && n_neighbours && top + n_neighbours > IVFPQ_MAX_MIXED)
        return fail(IVFPQ_EUNSUPPORTED, "%s: %d alternatives and %d neighbours, together over %d", what, top, n_neighbours, (int)IVFPQ_MAX_MIXED);
    if (n_neighbours && !(weight > 0.f && weight < 1.f)) return fail(IVFPQ_EINVAL, "%s: weight must be above 0 and below 1", what);
    if (n == 0) return IVFPQ_OK;
    if (n_neighbours && (!d_neighbour_tokens || !d_neighbour_logprobs)) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    if ((d_targets == nullptr) != (d_logprobs == nullptr)) return fail(IVFPQ_EINVAL, "%s: targets and logprobs go together", what);
    if (top && (!d_top_tokens || !d_top_logprobs)) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    const int want = top ? top + n_neighbours : 0;
    if (int s = check_workspace(what, d_workspace, workspace_bytes, row_workspace(n, vocab, want))) return s;
    const RowsIn in = rows_in(d_logits, row_stride, vocab, temperature);
    const ScoreOut out{d_targets, Listed{d_neighbour_tokens, d_neighbour_logprobs, n_neighbours},
                       n_neighbours ? (float)std::log1p(-(double)weight) : 0.f, n_neighbours ? (float)std::log((double)weight) : 0.f, top, want,
                       d_logprobs, d_entropy, d_norms, d_top_tokens, d_top_logprobs};
    return with_value_type(dtype, [&](auto v) {
        using T = decltype(v);
        if (top) return launch_rows<T, RowMode::kScoreTop>(n, in, out, d_workspace, (hipStream_t)hip_stream);
        return launch_rows<T, RowMode::kScore>(n, in, out, d_workspace, (hipStream_t)hip_stream);
    });
}

int distill_forward(const RowsIn& in, int32_t dtype, int64_t n, const Listed& teacher, float* d_loss, float* d_norms,
                    void* d_workspace, hipStream_t stream) {
    const DistillOut out{teacher, d_loss, d_norms};
    return with_value_type(dtype, [&](auto v) {
        return launch_rows<decltype(v), RowMode::kDistill>(n, in, out, d_workspace, stream);
    });
}

int distill_gradient(const RowsIn& in, int32_t dtype, int64_t n, const Listed& teacher, const float* d_row_grads, const float* d_norms,
                     void* d_grad, int64_t grad_stride, hipStream_t stream) {
    GradIn g{};
    g.norms = d_norms;
    g.grad = d_grad;
    g.grad_stride = grad_stride;
    const DistillGrad how{teacher, d_row_grads};
    return with_value_type(dtype, [&](auto v) { return launch_gradient<decltype(v), false>(n, in, g, how, stream); });
}

template <class T, int THREADS, int HELD>
int launch_step(int64_t n, const RowsIn& in, const DistillGrad& how, float* d_loss, void* d_grad, int64_t grad_stride, hipStream_t stream) {
    hipLaunchKernelGGL((distill_step_kernel<T, THREADS, HELD>), dim3((unsigned)n), dim3(THREADS), 0, stream, in, how, d_loss, d_grad, (long long)grad_stride);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

int distill_step(const RowsIn& in, int32_t dtype, int64_t n, const Listed& teacher, const float* d_row_grads, float* d_loss, void* d_grad,
                 int64_t grad_stride, hipStream_t stream) {
    const DistillGrad how{teacher, d_row_grads};
    const int64_t chunks = ((int64_t)in.vocab * value_bytes(dtype) + 15) / 16;
    return with_value_type(dtype, [&](auto v) {
        using T = decltype(v);
        if (chunks <= 4 * 256) return launch_step<T, 256, 4>(n, in, how, d_loss, d_grad, grad_stride, stream);      // fewer registers: twice the rows at once
        if (chunks <= kHeldChunks * 256) return launch_step<T, 256, kHeldChunks>(n, in, how, d_loss, d_grad, grad_stride, stream);
        if (chunks <= kHeldChunks * 512) return launch_step<T, 512, kHeldChunks>(n, in, how, d_loss, d_grad, grad_stride, stream);
        return launch_step<T, 1024, kHeldChunks>(n, in, how, d_loss, d_grad, grad_stride, stream);
    });
}

size_t distill_scratch(int64_t n, int32_t vocab) {
    if (n < 1 || n > kMostRows) return 0;
    return align_up((size_t)n * 2 * sizeof(float)) + row_workspace(n, vocab, 0);      // norms of a step, then the split rows
}

}  // namespace

extern "C" {

size_t ivfpq_token_logprobs_workspace_bytes(int64_t n, int32_t vocab, int32_t top, int32_t n_neighbours) {
    if (top < 0 || top > IVFPQ_MAX_TOP || n_neighbours < 0 || n_neighbours > IVFPQ_MAX_LISTED) return 0;
    return row_workspace(n, vocab, top ? std::min<int>(top + n_neighbours, IVFPQ_MAX_MIXED) : 0);
}

int ivfpq_token_logprobs(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride, const int32_t* d_targets,
                         float temperature, int32_t top, const int32_t* d_neighbour_tokens, const float* d_neighbour_logprobs,
                         int32_t n_neighbours, float weight, float* d_logprobs, float* d_entropy, float* d_norms,
                         int32_t* d_top_tokens, float* d_top_logprobs, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    return guarded("ivfpq_token_logprobs", [&] {
        return token_logprobs(d_logits, dtype, n, vocab, row_stride, d_targets, temperature, top, d_neighbour_tokens, d_neighbour_logprobs,
                              n_neighbours, weight, d_logprobs, d_entropy, d_norms, d_top_tokens, d_top_logprobs, d_workspace,
                              workspace_bytes, hip_stream);
    });
}

int ivfpq_token_logprobs_backward(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                                  const int32_t* d_targets, float temperature, const float* d_norms, const float* d_entropy,
                                  const float* d_grad_logprobs, const float* d_grad_entropy, void* d_grad, int64_t grad_stride,
                                  void* hip_stream) {
    return guarded("ivfpq_token_logprobs_backward", [&] {
        const char* what = "ivfpq_token_logprobs_backward";
        if (int s = check_rows(what, d_logits, dtype, n, vocab, row_stride, temperature)) return s;
        if (int s = check_grad(what, d_logits, row_stride, d_grad, dtype, n, vocab, grad_stride)) return s;
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_norms) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        if (!d_grad_logprobs && !d_grad_entropy) return fail(IVFPQ_EINVAL, "%s: neither gradient is given", what);
        if (d_grad_logprobs && !d_targets) return fail(IVFPQ_EINVAL, "%s: gradients of log-probabilities without targets", what);
        if (d_grad_entropy && !d_entropy) return fail(IVFPQ_EINVAL, "%s: gradients of entropies without entropies", what);
        const RowsIn in = rows_in(d_logits, row_stride, vocab, temperature);
        GradIn g{};
        g.norms = d_norms;
        g.grad = d_grad;
        g.grad_stride = grad_stride;
        const PolicyGrad how{d_targets, d_entropy, d_grad_logprobs, d_grad_entropy};
        return with_value_type(dtype, [&](auto v) {
            using T = decltype(v);
            if (d_grad_entropy) return launch_gradient<T, true>(n, in, g, how, (hipStream_t)hip_stream);
            return launch_gradient<T, false>(n, in, g, how, (hipStream_t)hip_stream);
        });
    });
}

size_t ivfpq_distill_topk_workspace_bytes(int64_t n, int32_t vocab) { return distill_scratch(n, vocab); }

int ivfpq_distill_topk(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride, const int32_t* d_teacher_tokens,
                       const float* d_teacher_logits, int32_t k, float temperature, float* d_loss, float* d_norms, void* d_workspace,
                       size_t workspace_bytes, void* hip_stream) {
    return guarded("ivfpq_distill_topk", [&] {
        const char* what = "ivfpq_distill_topk";
        if (int s = check_rows(what, d_logits, dtype, n, vocab, row_stride, temperature)) return s;
        if (int s = check_listed(what, d_teacher_tokens, d_teacher_logits, n, k)) return s;
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_loss || !d_norms) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        if (int s = check_workspace(what, d_workspace, workspace_bytes, distill_scratch(n, vocab))) return s;
        void* split = (char*)d_workspace + align_up((size_t)n * 2 * sizeof(float));
        return distill_forward(rows_in(d_logits, row_stride, vocab, temperature), dtype, n, Listed{d_teacher_tokens, d_teacher_logits, k},
                               d_loss, d_norms, split, (hipStream_t)hip_stream);
    });
}

int ivfpq_distill_topk_backward(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride, const float* d_norms,
                                const int32_t* d_teacher_tokens, const float* d_teacher_logits, int32_t k, float temperature,
                                const float* d_row_grads, void* d_grad, int64_t grad_stride, void* hip_stream) {
    return guarded("ivfpq_distill_topk_backward", [&] {
        const char* what = "ivfpq_distill_topk_backward";
        if (int s = check_rows(what, d_logits, dtype, n, vocab, row_stride, temperature)) return s;
        if (int s = check_listed(what, d_teacher_tokens, d_teacher_logits, n, k)) return s;
        if (int s = check_grad(what, d_logits, row_stride, d_grad, dtype, n, vocab, grad_stride)) return s;
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_norms) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        return distill_gradient(rows_in(d_logits, row_stride, vocab, temperature), dtype, n, Listed{d_teacher_tokens, d_teacher_logits, k},
                                d_row_grads, d_norms, d_grad, grad_stride, (hipStream_t)hip_stream);
    });
}

int ivfpq_distill_topk_step(const void* d_logits, int32_t dtype, int64_t n, int32_t vocab, int64_t row_stride,
                            const int32_t* d_teacher_tokens, const float* d_teacher_logits, int32_t k, float temperature,
                            const float* d_row_grads, float* d_loss, void* d_grad, int64_t grad_stride, void* d_workspace,
                            size_t workspace_bytes, void* hip_stream) {
    return guarded("ivfpq_distill_topk_step", [&] {
        const char* what = "ivfpq_distill_topk_step";
        if (int s = check_rows(what, d_logits, dtype, n, vocab, row_stride, temperature)) return s;
        if (int s = check_listed(what, d_teacher_tokens, d_teacher_logits, n, k)) return s;
        if (int s = check_grad(what, d_logits, row_stride, d_grad, dtype, n, vocab, grad_stride)) return s;
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_loss) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        if (int s = check_workspace(what, d_workspace, workspace_bytes, distill_scratch(n, vocab))) return s;
        float* norms = (float*)d_workspace;
        void* split = (char*)d_workspace + align_up((size_t)n * 2 * sizeof(float));
        const RowsIn in = rows_in(d_logits, row_stride, vocab, temperature);
        const Listed teacher{d_teacher_tokens, d_teacher_logits, k};
        const hipStream_t stream = (hipStream_t)hip_stream;
        if (step_in_registers(n, vocab, value_bytes(dtype)))
            return distill_step(in, dtype, n, teacher, d_row_grads, d_loss, d_grad, grad_stride, stream);
        if (int s = distill_forward(in, dtype, n, teacher, d_loss, norms, split, stream)) return s;
        return distill_gradient(in, dtype, n, teacher, d_row_grads, norms, d_grad, grad_stride, stream);
    });
}

}  // extern "C"
