// Which kernels the language-model calls take, by sizes alone.  Plain C++, so that a test can ask the same rules.
#pragma once

#include <cstdint>

namespace ivfpq {

// The kernel of an 8-bit product of m and n rows of k codes: `tiles` of rows x columns outputs a workgroup, or strips of that many a wave.
//
// Few rows of a, or few outputs: the tiles of 128 x 128 would leave most of the GPU idle (measured with k = 4096, a of 32 rows: n = 4,000
// 8.6 against 20 us, 16,000 19 against 23, 32,768 34 against 25; of 64 rows: n = 8,000 17 against 23, 32,768 52 against 27).
// Two blocks of b a wave where enough waves are left (32 rows: n = 32,768 34 against 46 us, 4,000 11 against 8.6).
struct ProductKernel {
    bool tiles;
    int rows, columns;
};
inline ProductKernel product_kernel(int64_t m, int64_t n, int k) {
    const int64_t strips = (m <= 32 ? 2 : (m + 63) / 64 * 4) * n;       // blocks of 16 rows that the waves would multiply, times n
    if (m <= 16 || strips <= 40000) return {false, m <= 16 ? 16 : m <= 32 ? 32 : 64, n >= 8192 ? 32 : 16};
    // tiles of 256 x 256 where the GPU has one for every CU (1,000 x 30,000, k = 900: 63 us against 83; 512 x 32,768, k = 4,096: 75 against 86),
    // but for sums of few slices, whose time is the stores: more, smaller workgroups overlap them (777 x 100,003, k = 96: 75 against 87)
    if (k > 256 && (m + 255) / 256 * ((n + 255) / 256) >= 256) return {true, 256, 256};
    return {true, 128, 128};
}

}  // namespace ivfpq
