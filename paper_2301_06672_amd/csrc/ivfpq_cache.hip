// A paged cache of keys and values: rows of a pass rotated and put to their places (ivfpq_cache_append), the kept ones moved
// up behind each other (ivfpq_cache_keep).
//
// A pair (a, b) of components at position p turns by p f: amplitude (a cos - b sin, b cos + a sin).  p f is a product of 64 bits, and
// what is left of it modulo 2 pi fits 32: an angle of 10^6 would be off by 0.03 in fp32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_cache.hpp"

using namespace ivfpq;

namespace {

struct AppendIn {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    void *q_out, *k_cache, *v_cache;
    const int* depths;                // [n][m] or null
    const float* inv_freq;            // [rotated / 2]
    int heads, rotated, interleaved, granules;
    bool q_pieces, k_pieces, v_pieces; // rows are 16-byte aligned
    float amplitude;
    Pages at;
};

// 8 consecutive values of a row, widened
template <class T>
__device__ inline void load8(const T* p, bool pieces, float (&x)[8]) {
    if (pieces) {
        constexpr int VEC = Chunk<T>::VEC;
#pragma unroll
        for (int i = 0; i < 8 / VEC; ++i) {
            Chunk<T> c;
            c.bits = reinterpret_cast<const uint4*>(p)[i];
            float part[VEC];
            c.widen(part);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[i * VEC + j] = part[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
    }
}

constexpr int kAppendThreads = 256, kAppendAtOnce = 2;

// One workgroup for the rows whose places are one granule of 8: their values go to the cache as whole 16-byte pieces, and an angle is
// formed once for all heads.  Bound by HBM with prompts (6,552 rows of 32 + 2 x 8 heads of 128, 161 MB in and out: 47 us, and 35 where the last-level cache holds
// them; a copy of that takes 34.  One piece at once 50 and 38, four 68 and 48; divisions of indexes in the loop 56 and 45), by latency with single tokens (64 of
// them 6 us).
template <class T, class C>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(AppendIn in) {
    __shared__ float turns[8][kMostHead];           // cos, then sin, of each pair
    const int tid = threadIdx.x, d = in.at.d, m = in.at.m, kv_heads = in.at.kv_heads;
    const long long s = blockIdx.x / in.granules;
    const int len = in.at.len(s), count = in.at.count(s);
    const long long granule = (len >> 3) + (long long)(blockIdx.x % in.granules);
    // rows [first, last) of the granule's places; place 8 * granule + i holds row base + i
    const long long base = granule * 8 - len;
    const int first = (int)max(base, 0ll), used = (int)min(base + 8, (long long)count), all = (int)min(base + 8, (long long)m);
    if (first >= all) return;
    const int pieces = d / 8;                       // of a head
    const int page = used > first ? in.at.page_of(s, granule * 8) : -1;
    const int off = (int)(granule * 8) & (in.at.page() - 1);
    C* k_page = (C*)in.k_cache + (page < 0 ? 0 : page) * in.at.page_values();
    C* v_page = (C*)in.v_cache + (page < 0 ? 0 : page) * in.at.page_values();

    // values: 8 components of the granule's rows a thread, turned over in registers
    for (int i = tid; i < kv_heads * pieces && page >= 0; i += kAppendThreads) {
        const int head = i / pieces, c = i % pieces * 8;
        C* to = v_page + (((long long)head << in.at.shift) + off) * d + c * 8;
        const T* x = (const T*)in.v + (s * m + base) * in.v_stride + (long long)head * d + c;
        if (used - first == 8) {
            C held[8][8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                float a[8];
                load8(x + r * in.v_stride, in.v_pieces, a);
#pragma unroll
                for (int j = 0; j < 8; ++j) held[j][r] = (C)a[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                typedef C out_t __attribute__((ext_vector_type(8)));
                out_t y;
#pragma unroll
                for (int r = 0; r < 8; ++r) y[r] = held[j][r];
                *reinterpret_cast<out_t*>(to + j * 8) = y;
            }
        } else {
            for (int row = first; row < used; ++row) {
                float a[8];
                load8(x + (row - base) * in.v_stride, in.v_pieces, a);
#pragma unroll
                for (int j = 0; j < 8; ++j) to[j * 8 + (row - base)] = (C)a[j];
            }
        }
    }

    // angles
    const int half = in.rotated / 2;
    for (int i = tid; i < (used - first) * half; i += kAppendThreads) {
        const int row = first + i / half, pair = i % half;
        const double position = (double)len + (double)(in.depths ? in.depths[s * m + row] : row);
        double turn = position * (double)in.inv_freq[pair] * 0.15915494309189535;           // of 2 pi
        turn -= rint(turn);
        float sine, cosine;
        sincosf((float)(turn * 6.283185307179586), &sine, &cosine);
        turns[row - base][pair] = cosine * in.amplitude;
        turns[row - base][half + pair] = sine * in.amplitude;
    }
    __syncthreads();

    // queries, then keys: a piece of 8 components a thread, with the one that it turns with where they lie apart, and kAppendAtOnce of those loaded at once.  A
    // thread has the same components of other heads each time: divisions of every index would take as long as the memory.
    typedef C out_t __attribute__((ext_vector_type(8)));
    const bool apart = !in.interleaved && half > 0 && half % 8 == 0;
    const int units = pieces - (apart ? half / 8 : 0), all_heads = in.heads + kv_heads, at_once = kAppendThreads / units;
    int c = tid % units * 8, next_row = first, next_head = tid / units;
    const bool two = apart && c < half;
    if (apart && !two) c += half;
    if (next_head >= at_once) return;
    while (next_row < all) {
        int rows[kAppendAtOnce], heads[kAppendAtOnce];
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            while (next_head >= all_heads && next_row < all) {
                next_head -= all_heads;
                ++next_row;
            }
            rows[u] = next_row;
            heads[u] = next_head;
            next_head += at_once;
        }
        float a[kAppendAtOnce][8], b[kAppendAtOnce][8];
        const auto source = [&](int row, int head) {
            const long long flat = s * m + row;
            return head < in.heads ? (const T*)in.q + flat * in.q_stride + (long long)head * d : (const T*)in.k + flat * in.k_stride + (long long)(head - in.heads) * d;
        };
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            const int row = rows[u], head = heads[u];
            if (row >= used || (head >= in.heads && page < 0)) continue;
            const bool whole = head < in.heads ? in.q_pieces : in.k_pieces;
            const T* x = source(row, head) + c;
            load8(x, whole, a[u]);
            if (two) load8(x + half, whole, b[u]);
        }
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            const int row = rows[u], head = heads[u];
            const bool query = head < in.heads, used_row = row < used;
            if (row >= all || (!query && (!used_row || page < 0))) continue;
            C* to = query ? (C*)in.q_out + ((s * m + row) * in.heads + head) * d + c : k_page + (((long long)(head - in.heads) << in.at.shift) + off + (row - base)) * d + c;
            out_t y, z;
            if (!used_row) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = z[j] = (C)0.f;
            } else {
                const float* turn = turns[row - base];
                if (two) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float cosine = turn[c + j], sine = turn[half + c + j], p = a[u][j], r = b[u][j];
                        a[u][j] = p * cosine - r * sine;
                        z[j] = (C)(r * cosine + p * sine);
                    }
                } else if (apart || c >= in.rotated) {
                } else if (in.interleaved) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const int pair = (c + j) / 2;
                        if (c + j < in.rotated) {
                            const float cosine = turn[pair], sine = turn[half + pair], p = a[u][j], r = a[u][j + 1];
                            a[u][j] = p * cosine - r * sine;
                            a[u][j + 1] = r * cosine + p * sine;
                        }
                    }
                } else {
                    const T* x = source(row, head);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = c + j;
                        if (e >= in.rotated) continue;
                        const int pair = e < half ? e : e - half;
                        const float other = (float)x[e < half ? e + half : e - half], cosine = turn[pair], sine = turn[half + pair];
                        a[u][j] = e < half ? a[u][j] * cosine - other * sine : a[u][j] * cosine + other * sine;
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = (C)a[u][j];
            }
            *reinterpret_cast<out_t*>(to) = y;
            if (two) *reinterpret_cast<out_t*>(to + half) = z;
        }
    }
}

struct KeepIn {
    uint16_t *k_cache, *v_cache;
    const int *path, *kept;           // [n][m], [n]
    int layers;
    Pages at;
};

constexpr int kKeepThreads = 256, kKeepBatch = 8;

// Where a kept row lies and goes to: page, and place in the page.
struct Move {
    int from, from_place, to, to_place;
};

// A thread moves a component of a head in a layer through all kept rows: neighbours read values 16 bytes apart and keys side by side.  (8 components a thread, keys
// as whole pieces: 14 us instead of 4 for 5 rows in 32 layers of 8 heads of 128, 43 instead of 19 for 64 sequences' in 16.)  The row that comes to place i lies behind
// it and before the sources of later places, so what a batch overwrites is never read by a later one; within a batch everything is read first.  Where
// rows lie is looked up for the whole workgroup at once, and rows that stay are left out, so that a batch is loaded without a branch.  Bound by
// the lines that values of single places lie in, 8 times what moves.
__global__ __launch_bounds__(kKeepThreads) void cache_keep_kernel(KeepIn in) {
    __shared__ Move moves[kKeepThreads];
    __shared__ int found[kKeepThreads / 64];
    const int d = in.at.d, m = in.at.m, per = in.at.kv_heads * d, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long s = blockIdx.y;
    const int kept = min(max(in.kept[s], 0), m);
    const long long len = in.at.len(s);
    const unsigned i = blockIdx.x * kKeepThreads + tid;         // 2^12 layers of 2^12 heads of 2^8 components at most, and what fills up the last workgroup
    const bool mine = i < (unsigned long long)per * in.layers;
    const unsigned layer = mine ? i / per : 0, rest = mine ? i - layer * per : 0, head = rest / d, c = rest % d;
    const long long layer_base = layer * (in.at.n_pages * in.at.page_values());
    const long long head_base = ((long long)head << in.at.shift) * d;
    uint16_t* const keys_at = in.k_cache + layer_base + head_base + c;
    uint16_t* const values_at = in.v_cache + layer_base + head_base + c * 8;
    const int* path = in.path + s * m;
    const int in_page = in.at.page() - 1;
    for (int base = 0; base < kept; base += kKeepThreads) {
        Move move{-1, 0, -1, 0};
        if (base + tid < kept) {
            const int row = path[base + tid];
            if (row > base + tid && row < m) {
                move = Move{in.at.page_of(s, len + row), (int)(len + row) & in_page, in.at.page_of(s, len + base + tid), (int)(len + base + tid) & in_page};
            }
        }
        const bool moves_so = move.from >= 0 && move.to >= 0;
        const uint64_t mask = __ballot(moves_so);
        __syncthreads();                                        // of the rows before
        if (lane == 0) found[wave] = __popcll(mask);
        __syncthreads();
        int count = 0, at = 0;
#pragma unroll
        for (int w = 0; w < kKeepThreads / 64; ++w) {
            if (w == wave) at = count + __popcll(mask & (((uint64_t)1 << lane) - 1));
            count += found[w];
        }
        if (moves_so) moves[at] = move;
        __syncthreads();
        if (!mine) continue;
        for (int first = 0; first < count; first += kKeepBatch) {
            uint16_t keys[kKeepBatch], values[kKeepBatch];
#pragma unroll
            for (int j = 0; j < kKeepBatch; ++j) {
                const Move x = moves[min(first + j, count - 1)];
                const long long from = x.from * in.at.page_values();
                keys[j] = keys_at[from + x.from_place * d];
                values[j] = values_at[from + (x.from_place & ~7) * d + (x.from_place & 7)];
            }
#pragma unroll
            for (int j = 0; j < kKeepBatch; ++j) {
                if (first + j >= count) break;
                const Move x = moves[first + j];
                const long long to = x.to * in.at.page_values();
                keys_at[to + x.to_place * d] = keys[j];
                values_at[to + (x.to_place & ~7) * d + (x.to_place & 7)] = values[j];
            }
        }
    }
}

template <class T, class C>
int launch_append(const AppendIn& in, int64_t n, hipStream_t stream) {
    hipLaunchKernelGGL((cache_append_kernel<T, C>), dim3((unsigned)(n * in.granules)), dim3(kAppendThreads), 0, stream, in);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

}  // namespace

extern "C" {

int ivfpq_cache_append(const void* d_q, int64_t q_stride, int32_t heads, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                       int32_t dtype, int64_t n, int32_t m, const int32_t* d_depths, const int32_t* d_counts, const float* d_inv_freq,
                       int32_t rotated, int32_t interleaved, float amplitude, void* d_q_out, void* d_k_cache, void* d_v_cache,
                       int32_t cache_dtype, int64_t n_pages, int32_t kv_heads, int32_t page, int32_t d, const int32_t* d_pages,
                       int32_t max_pages, const int32_t* d_lens, void* hip_stream) {
    return guarded("ivfpq_cache_append", [&] {
        const char* what = "ivfpq_cache_append";
        if (int rc = check_cache(what, d_k_cache, d_v_cache, cache_dtype, n_pages, kv_heads, page, d, d_pages, max_pages, d_lens, n, m)) return rc;
        if (!known_dtype(dtype)) return fail(IVFPQ_EINVAL, "%s: unknown dtype %d", what, dtype);
        if (dtype != IVFPQ_VALUES_FP32 && dtype != cache_dtype) return fail(IVFPQ_EINVAL, "%s: 16-bit rows are of the cache's dtype", what);
        if (m > kMostChain) return fail(IVFPQ_EUNSUPPORTED, "%s: m=%d (limit 2^20 rows)", what, m);
        if (heads < 0 || (heads > 0) != (d_q != nullptr) || (heads > 0) != (d_q_out != nullptr))
            return fail(IVFPQ_EINVAL, "%s: heads, queries and their output come together", what);
        if (heads > 65536) return fail(IVFPQ_EUNSUPPORTED, "%s: heads=%d (limit 65536)", what, heads);
        if (rotated < 0 || rotated > d || rotated % 2) return fail(IVFPQ_EINVAL, "%s: rotated=%d is no even number up to d=%d", what, rotated, d);
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_k || !d_v || (rotated > 0 && !d_inv_freq)) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        const int64_t rows = n * m, vb = value_bytes(dtype);
        if (rows > 1 && (k_stride < (int64_t)kv_heads * d || v_stride < (int64_t)kv_heads * d || (heads && q_stride < (int64_t)heads * d)))
            return fail(IVFPQ_EINVAL, "%s: a row stride below the row's values", what);
        if ((uintptr_t)d_k % vb || (uintptr_t)d_v % vb || (uintptr_t)d_q % vb || (uintptr_t)d_q_out % 16)
            return fail(IVFPQ_EINVAL, "%s: rows are not aligned to their type, or the queries' output not to 16 bytes", what);
        const auto whole = [&](const void* p, int64_t stride) { return (uintptr_t)p % 16 == 0 && (rows == 1 || stride * vb % 16 == 0); };
        AppendIn in{d_q, d_k, d_v, q_stride, k_stride, v_stride, d_q_out, d_k_cache, d_v_cache, d_depths, d_inv_freq, heads, rotated, interleaved,
                    (int)(((int64_t)m + 7 + 7) / 8),           // a pass may begin inside of a granule
                    whole(d_q, q_stride), whole(d_k, k_stride), whole(d_v, v_stride), amplitude,
                    pages_in(d_pages, max_pages, d_lens, d_counts, n_pages, kv_heads, page, d, m)};
        if (m == 1) in.granules = 1;
        const hipStream_t stream = (hipStream_t)hip_stream;
        return with_value_type(dtype, [&](auto t) {
            using T = decltype(t);
            if (cache_dtype == IVFPQ_VALUES_FP16) {
                if constexpr (!std::is_same<T, bf16_t>::value) return launch_append<T, half_t>(in, n, stream);
            } else {
                if constexpr (!std::is_same<T, half_t>::value) return launch_append<T, bf16_t>(in, n, stream);
            }
            return (int)IVFPQ_EINVAL;
        });
    });
}

int ivfpq_cache_keep(void* d_k_cache, void* d_v_cache, int32_t cache_dtype, int32_t layers, int64_t n_pages, int32_t kv_heads, int32_t page,
                     int32_t d, const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, int64_t n, int32_t m, const int32_t* d_path,
                     const int32_t* d_kept, void* hip_stream) {
    return guarded("ivfpq_cache_keep", [&] {
        const char* what = "ivfpq_cache_keep";
        if (int rc = check_cache(what, d_k_cache, d_v_cache, cache_dtype, n_pages, kv_heads, page, d, d_pages, max_pages, d_lens, n, m)) return rc;
        if (layers < 1 || layers > 4096) return fail(IVFPQ_EINVAL, "%s: layers=%d outside [1, 4096]", what, layers);
        if ((int64_t)layers * kv_heads * d > ((int64_t)1 << 31)) return fail(IVFPQ_EUNSUPPORTED, "%s: layers=%d kv_heads=%d d=%d (limit 2^31 components)", what, layers, kv_heads, d);
        if (m > kMostChain) return fail(IVFPQ_EUNSUPPORTED, "%s: m=%d (limit 2^20 rows)", what, m);
        if (n == 0) return (int)IVFPQ_OK;
        if (!d_path || !d_kept) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
        const KeepIn whole{(uint16_t*)d_k_cache, (uint16_t*)d_v_cache, d_path, d_kept, layers, pages_in(d_pages, max_pages, d_lens, nullptr, n_pages, kv_heads, page, d, m)};
        const int64_t items = (int64_t)layers * kv_heads * d;
        const int64_t wide = (items + kKeepThreads - 1) / kKeepThreads, kPiece = std::max<int64_t>(1, std::min<int64_t>(32768, ((int64_t)1 << 23) / wide));      // sequences of a launch of fewer than 2^32 threads
        for (int64_t at = 0; at < n; at += kPiece) {
            KeepIn in = whole;
            in.path += at * m;
            in.kept += at;
            in.at.lens += at;
            in.at.pages += at * max_pages;
            hipLaunchKernelGGL(cache_keep_kernel, dim3((unsigned)wide, (unsigned)std::min(kPiece, n - at)),
                               dim3(kKeepThreads), 0, (hipStream_t)hip_stream, in);
            HIP_TRY(hipGetLastError());
        }
        return (int)IVFPQ_OK;
    });
}

}  // extern "C"
