// Rows as signed 8-bit codes with a scale each, and the product of two sets of such rows on the matrix cores:
//   out[i][j] = (sa_i sb_j) sum_c a_ic b_jc + bias_j.
// The sums are exact in int32 (at most 2^16 products of at most 2^14), so neither the order of summation nor the kernel
// chosen shows in the result.  Two kernels: skinny_kernel for few rows of a, bound by reading b once, and tile_kernel, bound by the
// matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ivfpq_hip_util.hpp"
#include "ivfpq_language_rules.hpp"
#include "ivfpq_values.hpp"

using namespace ivfpq;

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

// ---- rows to codes

constexpr int kHeld = 4;                  // chunks a thread holds between the pass for the scale and the pass for the codes

// LANES threads a row, 256 / LANES rows a workgroup (LANES 64 or 256).  Reads every row once (rows over kHeld chunks a thread:
// the rest a second time, from the caches).  The scale is a maximum, so a row has to be seen before its first code: it is held in
// registers in between.  2,048 x 4,096 bf16: 11 us (25 MB, 2.3 TB/s: a chain of load, maximum, division, store); one such row 4 us.
template <class T, int LANES>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* __restrict__ rows, long long n, int d, long long stride,
                                                            int8_t* __restrict__ codes, long long code_stride, float* __restrict__ scales) {
    constexpr int VEC = Chunk<T>::VEC, ROWS = 256 / LANES;
    __shared__ uint32_t wave_most[4];
    const int lane = threadIdx.x % LANES;
    const long long r = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
    const bool live = r < n;
    const RowChunks<T> row(rows, live ? r : 0, stride, d);
    const int n_chunks = live ? row.count() : 0;
    // magnitudes as integers: a NaN is the largest, then infinity
    uint32_t most = 0;
    auto widest = [&](const Chunk<T>& k) {
        float x[VEC];
        k.widen(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) most = max(most, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    };
    Chunk<T> held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (lane + i * LANES < n_chunks) held[i] = row.load(lane + i * LANES, 0.f);
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (lane + i * LANES < n_chunks) widest(held[i]);
    for (int c = lane + kHeld * LANES; c < n_chunks; c += LANES) widest(row.load(c, 0.f));
    for (int off = 32; off; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if constexpr (LANES == 256) {
        if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3]));
    }
    if (!live) return;
    const bool odd = most >= 0x7F800000u;
    const float scale = odd ? __uint_as_float(0x7FC00000u) : __uint_as_float(most) / 127.f;
    if (lane == 0) scales[r] = scale;
    int8_t* to = codes + r * code_stride;
    const bool zero = odd || scale == 0.f;
    auto put = [&](const Chunk<T>& k, int c) {
        float x[VEC];
        k.widen(x);
        int q[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            q[j] = zero ? 0 : (int)fminf(fmaxf(rintf(x[j] / scale), -127.f), 127.f);
        const int at = c * VEC - row.lead;
        if (row.whole(c) && ((reinterpret_cast<uintptr_t>(to) + at) & 3) == 0) {
#pragma unroll
            for (int j = 0; j < VEC; j += 4)
                *reinterpret_cast<uint32_t*>(to + at + j) = (q[j] & 255) | (q[j + 1] & 255) << 8 | (q[j + 2] & 255) << 16 | (uint32_t)(q[j + 3] & 255) << 24;
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (at + j >= 0 && at + j < d) to[at + j] = (int8_t)q[j];
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
        if (lane + i * LANES < n_chunks) put(held[i], lane + i * LANES);
    for (int c = lane + kHeld * LANES; c < n_chunks; c += LANES) put(row.load(c, 0.f), c);
    for (long long c = d + lane; c < code_stride; c += LANES) to[c] = 0;
}

// ---- products

struct Product {
    const int8_t *a, *b;
    long long a_stride, b_stride, out_stride;
    const float *a_scales, *b_scales, *bias;
    void* out;
    int m, n, k;
    bool aligned;                     // every row of out begins at a multiple of 64 bytes
};

__device__ inline float scaled(int acc, float sa, float sb, float bias) { return (sa * sb) * (float)acc + bias; }

// Bytes [at, at + 16) of a row, 0 from k on: a sum takes nothing of what lies there.
__device__ inline intx4 masked16(const int8_t* row, int at, int k) {
    intx4 v = {0, 0, 0, 0};
    if (at >= k) return v;
    v = *reinterpret_cast<const intx4*>(row + at);
    if (at + 16 > k) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int left = k - at - 4 * w;               // bytes of this word that count
            const uint32_t keep = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
            v[w] &= (int)keep;
        }
    }
    return v;
}

// Few rows of a.  v_mfma_i32_16x16x64_i8: a wave has MT x NT blocks of 16 x 16; lane L brings row / column L % 16 and bytes
// [16 (L / 16), ...) of each 64; register v of lane L holds row 4 (L / 16) + v, column L % 16.  The operands come straight
// from memory in that layout (b is read once, a from the caches); the four waves of a workgroup take every fourth of the
// 128-byte lines of the rows and add up through the LDS.  Bound by reading b: 32,768 rows of 4,096 against one row 24 us where
// half of b is still in the last-level cache (two sets of weights in turn: 5.5 TB/s), 31 us where nothing is (eight in turn: 4.4 TB/s).
template <class T, int MT, int NT>
__global__ __launch_bounds__(256) void skinny_kernel(Product p) {
    __shared__ int sums[3][MT * NT * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j0 = blockIdx.x * 16 * NT, i0 = blockIdx.y * 16 * MT;
    const int part = 16 * (lane >> 4);
    const int8_t* a[MT];
    const int8_t* b[NT];
#pragma unroll
    for (int t = 0; t < MT; ++t) a[t] = p.a + (long long)min(i0 + 16 * t + (lane & 15), p.m - 1) * p.a_stride;
#pragma unroll
    for (int t = 0; t < NT; ++t) b[t] = p.b + (long long)min(j0 + 16 * t + (lane & 15), p.n - 1) * p.b_stride;
    intx4 acc[MT][NT] = {};
    const int lines = (p.k + 127) / 128, whole = p.k / 128;
    int line = wave;
    for (; line < whole; line += 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = line * 128 + h * 64 + part;
            intx4 va[MT], vb[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) vb[t] = *reinterpret_cast<const intx4*>(b[t] + at);
#pragma unroll
            for (int t = 0; t < MT; ++t) va[t] = *reinterpret_cast<const intx4*>(a[t] + at);
#pragma unroll
            for (int s = 0; s < MT; ++s)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[s][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(va[s], vb[t], acc[s][t], 0, 0, 0);
        }
    }
    if (line < lines) {                                    // the last line, cut at k
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = line * 128 + h * 64 + part;
            intx4 va[MT], vb[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) vb[t] = masked16(b[t], at, p.k);
#pragma unroll
            for (int t = 0; t < MT; ++t) va[t] = masked16(a[t], at, p.k);
#pragma unroll
            for (int s = 0; s < MT; ++s)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[s][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(va[s], vb[t], acc[s][t], 0, 0, 0);
        }
    }
    if (wave) {
#pragma unroll
        for (int s = 0; s < MT; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) sums[wave - 1][(s * NT + t) * 4 + v][lane] = acc[s][t][v];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int j = j0 + 16 * t + (lane & 15);
        if (j >= p.n) continue;
        const float sb = p.b_scales[j], bias = p.bias ? p.bias[j] : 0.f;
#pragma unroll
        for (int s = 0; s < MT; ++s)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = i0 + 16 * s + 4 * (lane >> 4) + v;
                const int at = (s * NT + t) * 4 + v;
                const int sum = acc[s][t][v] + sums[0][at][lane] + sums[1][at][lane] + sums[2][at][lane];
                if (i < p.m) reinterpret_cast<T*>(p.out)[i * p.out_stride + j] = (T)scaled(sum, p.a_scales[i], sb, bias);
            }
    }
}

// Many rows of a: a tile of BM x BN outputs a workgroup of WM x WN waves, operands through the LDS in slices of 128 bytes of
// the rows, two slices in turn: one is loaded straight into the LDS while the other is multiplied, one barrier a slice.
// v_mfma_i32_32x32x32_i8: lane L brings row / column L % 32 and bytes [16 (L / 32), ...) of each 32; register v of lane L
// holds row 8 (v / 4) + 4 (L / 32) + v % 4, column L % 32.  Two rows of 128 bytes cover the 64 banks of the LDS, so the 16-byte
// pieces of row r stand in the order piece ^ (r / 2 % 8): sixteen lanes that read one piece of sixteen rows use every bank
// once.  Pieces are addressed by 32-bit offsets made once a tile (64-bit products for every load: 325 against 308 us below).
// 2,048 x 32,768 bf16 results of 4,096 components: 273 to 282 us, 2.0 POP/s (the library's int8 product of that shape, without scales:
// 266 to 269); 8,192^3 484 us, 2.3 POP/s (440).  The matrix cores are 0.4 busy; a CU's LDS reads (0.75 of the products' time), its loads of
// the next slice and the products overlap between the two waves of a SIMD, and all of them wait for the slowest at the barrier
// of a slice.  Slices of 64 bytes, three of them ahead in four buffers: 343 against 308 us; slices begun at another place
// by every workgroup, against rows a power of two apart in one channel: no gain (323 against 325).
__device__ inline int piece_at(int row, int piece) { return piece ^ ((row >> 1) & 7); }

// Sums on their way out: rows of BN words and 8 more, which puts rows four apart into opposite halves of the banks
template <int BN> constexpr int kStagePitch = BN + 8;
template <int BN, int WM> constexpr size_t kStageBytes = (size_t)WM * 32 * kStagePitch<BN> * sizeof(int);

// 16 bytes a lane straight into the LDS, 1024 from `to` on in the order of the lanes
__device__ inline void load_piece(const int8_t* base, uint32_t offset, int8_t* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + offset), (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <class T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(Product p) {
    constexpr int WAVES = WM * WN, SM = BM / (32 * WM), SN = BN / (32 * WN);
    extern __shared__ int8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int tiles_n = (p.n + BN - 1) / BN;
    unsigned tile = blockIdx.x;
    // Rows of out that begin anywhere: the tiles of a row share the 64-byte pieces at their borders, which only one L2 can put
    // together.  Workgroups go to the eight XCDs in turn, so each XCD takes a range of consecutive tiles (777 x 100,003 fp32 results of 96
    // components: 78 against 111 us).  Aligned rows pass the caches by instead (2,048 x 32,768 bf16, k = 256: 77 against 85 us, k = 4,096: 268 against
    // 277; 777 x 100,032 fp32, k = 96: 69 against 71; 4,096 x 14,016 fp32, k = 256: 66 and 65).
    if (!p.aligned) {
        const unsigned each = gridDim.x / 8, more = gridDim.x % 8, xcd = blockIdx.x % 8;
        tile = xcd * each + min(xcd, more) + blockIdx.x / 8;
    }
    const int i0 = (int)(tile / (unsigned)tiles_n) * BM, j0 = (int)(tile % (unsigned)tiles_n) * BN;
    constexpr int SLICE = (BM + BN) * 128;
    // a wave loads eight rows of a slice at a time: lane L the piece that stands at L % 8 in row L / 8 of them
    const int sub = lane >> 3;
    const int slices = (p.k + 127) / 128;
    // where a lane's pieces begin, from the tile's first row (rows beyond the last one: the last one again)
    constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;
    const int8_t* from_a = p.a + i0 * p.a_stride;
    const int8_t* from_b = p.b + j0 * p.b_stride;
    uint32_t off_a[LA], off_b[LB];
#pragma unroll
    for (int t = 0; t < LA; ++t) {
        const int r = (t * WAVES + wave) * 8 + sub;
        off_a[t] = (uint32_t)min(r, p.m - 1 - i0) * (uint32_t)p.a_stride + piece_at(r, lane & 7) * 16;
    }
#pragma unroll
    for (int t = 0; t < LB; ++t) {
        const int r = (t * WAVES + wave) * 8 + sub;
        off_b[t] = (uint32_t)min(r, p.n - 1 - j0) * (uint32_t)p.b_stride + piece_at(r, lane & 7) * 16;
    }
    auto load_slice = [&](int s) {
        int8_t* to = lds + (s & 1) * SLICE + wave * 1024;
        const int k0 = s * 128;
        if (k0 + 128 <= p.k) {
#pragma unroll
            for (int t = 0; t < LA; ++t) load_piece(from_a + k0, off_a[t], to + t * WAVES * 1024);
#pragma unroll
            for (int t = 0; t < LB; ++t) load_piece(from_b + k0, off_b[t], to + BM * 128 + t * WAVES * 1024);
        } else {                                           // the last slice, cut at k
#pragma unroll
            for (int t = 0; t < LA; ++t) {
                const int at = piece_at((t * WAVES + wave) * 8 + sub, lane & 7) * 16;
                *reinterpret_cast<intx4*>(to + t * WAVES * 1024 + lane * 16) = masked16(from_a + off_a[t] - at, k0 + at, p.k);
            }
#pragma unroll
            for (int t = 0; t < LB; ++t) {
                const int at = piece_at((t * WAVES + wave) * 8 + sub, lane & 7) * 16;
                *reinterpret_cast<intx4*>(to + BM * 128 + t * WAVES * 1024 + lane * 16) = masked16(from_b + off_b[t] - at, k0 + at, p.k);
            }
        }
    };
    intx16 acc[SM][SN] = {};
    const int l32 = lane & 31, half = lane >> 5;
    load_slice(0);
    for (int s = 0; s < slices; ++s) {
        __syncthreads();
        if (s + 1 < slices) load_slice(s + 1);
        const int8_t* at = lds + (s & 1) * SLICE;
        const int8_t* at_a = at + (wm * SM * 32 + l32) * 128;
        const int8_t* at_b = at + (BM + wn * SN * 32 + l32) * 128;
        // the operands of a step are read while the step before it is multiplied
        intx4 va[2][SM], vb[2][SN];
        auto read = [&](int step) {
            const int stands = piece_at(l32, 2 * step + half) * 16;
#pragma unroll
            for (int t = 0; t < SM; ++t) va[step & 1][t] = *reinterpret_cast<const intx4*>(at_a + t * 32 * 128 + stands);
#pragma unroll
            for (int t = 0; t < SN; ++t) vb[step & 1][t] = *reinterpret_cast<const intx4*>(at_b + t * 32 * 128 + stands);
        };
        read(0);
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            if (step < 3) read(step + 1);
#pragma unroll
            for (int x = 0; x < SM; ++x)
#pragma unroll
                for (int y = 0; y < SN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(va[step & 1][x], vb[step & 1][y], acc[x][y], 0, 0, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, SM + SN, 0);           // the first step's reads, then a read behind every product
#pragma unroll
        for (int step = 0; step < 3; ++step) {
#pragma unroll
            for (int o = 0; o < SM + SN; ++o) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            if (SM * SN > SM + SN) __builtin_amdgcn_sched_group_barrier(0x008, SM * SN - SM - SN, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, SM * SN, 0);
    }
    // The sums pass through the LDS, 32 rows of every wave at a time, so that a thread scales and stores 16 bytes of a row and a
    // row of the tile is written in one piece.
    constexpr int VEC = 16 / sizeof(T), PER_ROW = BN / VEC, AT_ONCE = 64 * WAVES / PER_ROW;
    typedef T piece_t __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
    int* stage = reinterpret_cast<int*>(lds);
    const int col = (int)threadIdx.x % PER_ROW * VEC, j = j0 + col;
    float sb[VEC], bias[VEC];
#pragma unroll
    for (int o = 0; o < VEC; ++o) {
        sb[o] = j + o < p.n ? p.b_scales[j + o] : 0.f;
        bias[o] = p.bias && j + o < p.n ? p.bias[j + o] : 0.f;
    }
#pragma unroll
    for (int x = 0; x < SM; ++x) {
        __syncthreads();
#pragma unroll
        for (int y = 0; y < SN; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                stage[(wm * 32 + 8 * (v / 4) + 4 * half + v % 4) * kStagePitch<BN> + (wn * SN + y) * 32 + l32] = acc[x][y][v];
        __syncthreads();
#pragma unroll
        for (int r = (int)threadIdx.x / PER_ROW; r < WM * 32; r += AT_ONCE) {
            const int i = i0 + (r / 32 * SM + x) * 32 + r % 32;
            if (i >= p.m || j >= p.n) continue;
            const float sa = p.a_scales[i];
            T* out = reinterpret_cast<T*>(p.out) + i * p.out_stride + j;
            piece_t y;
#pragma unroll
            for (int o = 0; o < VEC; ++o) y[o] = (T)scaled(stage[r * kStagePitch<BN> + col + o], sa, sb[o], bias[o]);
            if (j + VEC <= p.n && p.aligned) __builtin_nontemporal_store(y, reinterpret_cast<piece_t*>(out));
            else if (j + VEC <= p.n) *reinterpret_cast<piece_t*>(out) = y;
            else
                for (int o = 0; j + o < p.n; ++o) out[o] = y[o];
        }
    }
}

template <class T, int MT, int NT>
int launch_skinny(const Product& p, hipStream_t stream) {
    const dim3 grid((unsigned)((p.n + 16 * NT - 1) / (16 * NT)), (unsigned)((p.m + 16 * MT - 1) / (16 * MT)));
    hipLaunchKernelGGL((skinny_kernel<T, MT, NT>), grid, dim3(256), 0, stream, p);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

template <class T, int BM, int BN, int WM, int WN>
int launch_tiles(const Product& p, hipStream_t stream) {
    const size_t lds = std::max((size_t)(p.k > 128 ? 2 : 1) * (BM + BN) * 128, kStageBytes<BN, WM>);
    const int64_t tiles = (int64_t)((p.m + BM - 1) / BM) * ((p.n + BN - 1) / BN);
    if (tiles * (64 * WM * WN) > 0xFFFFFFFFll) return fail(IVFPQ_EUNSUPPORTED, "ivfpq_q8_matmul: m=%d n=%d is over 2^32 threads", p.m, p.n);
    if (int s = allow_full_lds(tile_kernel<T, BM, BN, WM, WN>)) return s;
    hipLaunchKernelGGL((tile_kernel<T, BM, BN, WM, WN>), dim3((unsigned)tiles), dim3(64 * WM * WN), lds, stream, p);
    HIP_TRY(hipGetLastError());
    return IVFPQ_OK;
}

constexpr int64_t kPiece = 1 << 22;        // rows of one launch: fewer than 2^32 threads
constexpr int64_t kMostStride = 1 << 24;   // 255 of them and a piece's place in its line are a 32-bit offset from a tile's first row

template <class T>
int launch_product(const Product& p, hipStream_t stream) {
    const ProductKernel kernel = product_kernel(p.m, p.n, p.k);
    if (kernel.tiles) return kernel.rows == 256 ? launch_tiles<T, 256, 256, 2, 4>(p, stream) : launch_tiles<T, 128, 128, 2, 2>(p, stream);
    const bool wide = kernel.columns == 32;
    if (kernel.rows == 16) return wide ? launch_skinny<T, 1, 2>(p, stream) : launch_skinny<T, 1, 1>(p, stream);
    if (kernel.rows == 32) return wide ? launch_skinny<T, 2, 2>(p, stream) : launch_skinny<T, 2, 1>(p, stream);
    return wide ? launch_skinny<T, 4, 2>(p, stream) : launch_skinny<T, 4, 1>(p, stream);
}

int q8_matmul(const int8_t* d_a, int64_t a_stride, const float* d_a_scales, int64_t m, const int8_t* d_b, int64_t b_stride,
              const float* d_b_scales, int64_t n, int32_t k, const float* d_bias, void* d_out, int32_t out_dtype, int64_t out_stride,
              void* hip_stream) {
    const char* what = "ivfpq_q8_matmul";
    if (!known_dtype(out_dtype)) return fail(IVFPQ_EINVAL, "%s: unknown dtype %d", what, out_dtype);
    if (m < 0 || n < 0) return fail(IVFPQ_EINVAL, "%s: bad shape", what);
    if (k < 1 || k > IVFPQ_MAX_Q8_K) return fail(IVFPQ_EINVAL, "%s: k=%d outside [1, %d]", what, k, (int)IVFPQ_MAX_Q8_K);
    if (m == 0 || n == 0) return IVFPQ_OK;
    if (!d_a || !d_b || !d_a_scales || !d_b_scales || !d_out) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    const int64_t least = (k + 15) / 16 * 16;
    if (a_stride < least || a_stride % 16 || b_stride < least || b_stride % 16)
        return fail(IVFPQ_EINVAL, "%s: code strides %lld, %lld: multiples of 16 of at least %lld are needed", what, (long long)a_stride, (long long)b_stride, (long long)least);
    if ((m > 1 && a_stride > kMostStride) || (n > 1 && b_stride > kMostStride))
        return fail(IVFPQ_EUNSUPPORTED, "%s: code strides %lld, %lld (limit 2^24)", what, (long long)a_stride, (long long)b_stride);
    if (((uintptr_t)d_a | (uintptr_t)d_b) % 16) return fail(IVFPQ_EINVAL, "%s: codes are not aligned to 16 bytes", what);
    if ((uintptr_t)d_out % value_bytes(out_dtype)) return fail(IVFPQ_EINVAL, "%s: the output is not aligned to its type", what);
    if (m > 1 && out_stride < n) return fail(IVFPQ_EINVAL, "%s: output stride %lld below n=%lld", what, (long long)out_stride, (long long)n);
    const size_t vb = value_bytes(out_dtype);
    const bool aligned = ((uintptr_t)d_out | (m > 1 ? (size_t)out_stride * vb : 0)) % 64 == 0;
    for (int64_t i = 0; i < m; i += kPiece)
        for (int64_t j = 0; j < n; j += kPiece) {
            const Product p{d_a + i * a_stride, d_b + j * b_stride, a_stride, b_stride, out_stride, d_a_scales + i, d_b_scales + j,
                            d_bias ? d_bias + j : nullptr, (char*)d_out + (i * out_stride + j) * vb,
                            (int)std::min(kPiece, m - i), (int)std::min(kPiece, n - j), k, aligned};
            if (int s = with_value_type(out_dtype, [&](auto v) { return launch_product<decltype(v)>(p, (hipStream_t)hip_stream); })) return s;
        }
    return IVFPQ_OK;
}

int quantize_rows(const void* d_rows, int32_t dtype, int64_t n, int32_t d, int64_t row_stride, int8_t* d_codes, int64_t code_stride,
                  float* d_scales, void* hip_stream) {
    const char* what = "ivfpq_quantize_rows";
    if (!known_dtype(dtype)) return fail(IVFPQ_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (n < 0) return fail(IVFPQ_EINVAL, "%s: bad shape", what);
    if (d < 1 || d > IVFPQ_MAX_Q8_K) return fail(IVFPQ_EINVAL, "%s: d=%d outside [1, %d]", what, d, (int)IVFPQ_MAX_Q8_K);
    if (code_stride < d || (n > 1 && row_stride < d)) return fail(IVFPQ_EINVAL, "%s: a stride is below d=%d", what, d);
    if (n == 0) return IVFPQ_OK;
    if (!d_rows || !d_codes || !d_scales) return fail(IVFPQ_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)d_rows % value_bytes(dtype)) return fail(IVFPQ_EINVAL, "%s: rows are not aligned to their type", what);
    return with_value_type(dtype, [&](auto v) {
        using T = decltype(v);
        const hipStream_t stream = (hipStream_t)hip_stream;
        for (int64_t at = 0; at < n; at += kPiece) {
            const long long rows = std::min(kPiece, n - at);
            const void* from = (const T*)d_rows + at * row_stride;
            int8_t* codes = d_codes + at * code_stride;
            if (d <= 64 * kHeld * Chunk<T>::VEC)           // a wave holds the row
                hipLaunchKernelGGL((quantize_rows_kernel<T, 64>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, from, rows, d,
                                   (long long)row_stride, codes, (long long)code_stride, d_scales + at);
            else
                hipLaunchKernelGGL((quantize_rows_kernel<T, 256>), dim3((unsigned)rows), dim3(256), 0, stream, from, rows, d,
                                   (long long)row_stride, codes, (long long)code_stride, d_scales + at);
            HIP_TRY(hipGetLastError());
        }
        return (int)IVFPQ_OK;
    });
}

}  // namespace

extern "C" {

int ivfpq_quantize_rows(const void* d_rows, int32_t dtype, int64_t n, int32_t d, int64_t row_stride, int8_t* d_codes, int64_t code_stride,
                        float* d_scales, void* hip_stream) {
    return guarded("ivfpq_quantize_rows", [&] { return quantize_rows(d_rows, dtype, n, d, row_stride, d_codes, code_stride, d_scales, hip_stream); });
}

int ivfpq_q8_matmul(const int8_t* d_a, int64_t a_stride, const float* d_a_scales, int64_t m, const int8_t* d_b, int64_t b_stride,
                    const float* d_b_scales, int64_t n, int32_t k, const float* d_bias, void* d_out, int32_t out_dtype, int64_t out_stride,
                    void* hip_stream) {
    return guarded("ivfpq_q8_matmul", [&] {
        return q8_matmul(d_a, a_stride, d_a_scales, m, d_b, b_stride, d_b_scales, n, k, d_bias, d_out, out_dtype, out_stride, hip_stream);
    });
}

}  // extern "C"
