// A layer's paged cache of keys and values, and the rows of a pass over it: what the kernels take and what every call checks.
// Included by .hip translation units only; everything has internal linkage.
#pragma once

#include "ivfpq_values.hpp"

namespace {

constexpr int kMostHead = IVFPQ_MAX_HEAD;
constexpr int64_t kMostPlaces = ((int64_t)1 << 31) - ((int64_t)1 << 21);      // a place and a pass's rows behind it fit an int32
constexpr int kMostChain = 1 << 20;

// Places of sequence s are in the pages that its row of `pages` lists.
struct Pages {
    const int* pages;                 // [n][stride]
    const int* lens;                  // [n]
    const int* counts;                // [n] or null
    long long n_pages;
    int stride, most, shift;          // of which the first `most` are looked at; page = 1 << shift
    int kv_heads, d, m;
    __device__ inline int page() const { return 1 << shift; }
    __device__ inline int len(long long s) const { return max(lens[s], 0); }
    __device__ inline int count(long long s) const { return counts ? min(max(counts[s], 0), m) : m; }
    __device__ inline long long page_values() const { return ((long long)kv_heads * d) << shift; }
    // The page of a place that is not negative, or -1.
    __device__ inline int page_of(long long s, long long place) const {
        const long long i = place >> shift;
        if (i >= most) return -1;
        const int id = pages[s * stride + i];
        return id >= 0 && id < n_pages ? id : -1;
    }
};

// What is wrong with a cache and its pages, or IVFPQ_OK.
inline int check_cache(const char* what, const void* k_cache, const void* v_cache, int32_t cache_dtype, int64_t n_pages, int32_t kv_heads,
                       int32_t page, int32_t d, const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, int64_t n, int32_t m) {
    if (cache_dtype != IVFPQ_VALUES_FP16 && cache_dtype != IVFPQ_VALUES_BF16) return fail(IVFPQ_EINVAL, "%s: a cache's dtype is fp16 or bf16, got %d", what, cache_dtype);
    if (n < 0 || m < 1 || n_pages < 0 || kv_heads < 1 || max_pages < 0) return fail(IVFPQ_EINVAL, "%s: bad shape (n=%lld m=%d n_pages=%lld kv_heads=%d max_pages=%d)", what, (long long)n, m, (long long)n_pages, kv_heads, max_pages);
    if (page < 16 || page > 256 || (page & (page - 1))) return fail(IVFPQ_EINVAL, "%s: page=%d is no power of two from 16 to 256", what, page);
    if (d < 8 || d > kMostHead || d % 8) return fail(IVFPQ_EINVAL, "%s: d=%d is no multiple of 8 up to %d", what, d, kMostHead);
    if (kv_heads > 4096) return fail(IVFPQ_EUNSUPPORTED, "%s: kv_heads=%d (limit 4096)", what, kv_heads);
    if (n_pages > ((int64_t)1 << 31) - 1) return fail(IVFPQ_EUNSUPPORTED, "%s: n_pages=%lld (limit 2^31 - 1)", what, (long long)n_pages);
    if ((int64_t)max_pages * page >= kMostPlaces) return fail(IVFPQ_EUNSUPPORTED, "%s: %d pages of %d (limit 2^31 - 2^21 places)", what, max_pages, page);
    if (n > (1 << 20) || n * m > (1 << 24)) return fail(IVFPQ_EUNSUPPORTED, "%s: n=%lld m=%d (limits 2^20 sequences, 2^24 rows)", what, (long long)n, m);
    if (n > 0 && ((n_pages > 0 && (!k_cache || !v_cache)) || !d_lens || (max_pages > 0 && !d_pages))) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)k_cache % 16 || (uintptr_t)v_cache % 16) return fail(IVFPQ_EINVAL, "%s: a cache is not aligned to 16 bytes", what);
    return IVFPQ_OK;
}

inline Pages pages_in(const int32_t* d_pages, int32_t max_pages, const int32_t* d_lens, const int32_t* d_counts, int64_t n_pages, int32_t kv_heads,
                      int32_t page, int32_t d, int32_t m) {
    return Pages{d_pages, d_lens, d_counts, (long long)n_pages, max_pages, max_pages, __builtin_ctz((unsigned)page), kv_heads, d, m};
}

}  // namespace
