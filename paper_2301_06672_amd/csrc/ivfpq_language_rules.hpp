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

// Whether a distillation step holds every row in the registers of one workgroup (kHeldChunks pieces of 16 bytes a thread, up to 1,024 threads): one
// launch and one read of the logits instead of three and two, but a row in 1 of 256 compute units, where the split kernels take as many as there
// are.  One row's time grows with its values, whatever their type; 16-bit rows have up to 131,072 of them, fp32 rows 65,536.  us, registers / split,
// called one after the other from Python (where three launches take 19 us of the host) and replayed from a graph:
//   bf16 values            called    1 row        16           48           96           160          replayed   1            16           48           96           160
//   50,000                 13.8 / 19.1  14.0 / 19.3  15.5 / 19.0  18.9 / 20.1  20.7 / 25.5            12.0 / 12.0  13.4 / 14.3  15.6 / 17.7  19.5 / 20.7  21.1 / 25.8
//   65,536                 13.9 / 18.8  16.0 / 19.1  17.2 / 19.1  22.0 / 22.7  23.6 / 27.1            13.8 / 11.7  16.4 / 15.1  18.0 / 17.7  22.8 / 23.2  23.6 / 27.4
//   80,000                 15.8 / 18.9  18.1 / 19.1  19.6 / 19.1  23.1 / 25.0  24.8 / 29.3            15.6 / 11.9  18.6 / 15.5  20.1 / 18.3  23.5 / 25.3  25.0 / 29.7
//   100,000                18.3 / 18.9  21.1 / 19.2  24.6 / 19.6  26.9 / 25.6  28.2 / 33.3            17.7 / 11.9  21.2 / 16.4  25.3 / 20.0  27.2 / 26.0  28.8 / 33.9
//   131,072                24.0 / 18.8  24.9 / 19.0  30.6 / 22.5  32.3 / 28.8  34.3 / 39.1            23.5 / 12.4  25.3 / 16.3  30.7 / 23.1  32.5 / 29.0  34.9 / 39.7
//   fp32: 65,536           13.6 / 18.9  13.8 / 19.2  17.5 / 21.5  20.1 / 27.6  24.9 / 38.0            12.6 / 12.1  13.3 / 15.6  17.6 / 21.9  20.1 / 27.9  25.2 / 38.6
// 4,096 rows of 65,536 bf16 values: 266 / 372.  Where the two ways of calling disagree, which is for few 16-bit rows of over 50,000 values, rows stay
// split below 16 of them and held from there on.
constexpr int kHeldChunks = 16;
inline bool step_in_registers(int64_t n, int64_t vocab, int value_bytes) {
    if (vocab * value_bytes > (int64_t)16 * kHeldChunks * 1024) return false;
    if (n < 16) return value_bytes == 4 || vocab <= 50000;
    return vocab <= 80000 || n >= 112;
}

}  // namespace ivfpq
