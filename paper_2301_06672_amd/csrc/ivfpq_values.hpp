// Rows of fp32, fp16 or bf16 values for the logit and 8-bit kernels: widening, rounding, 16-byte chunks of a row of any
// alignment, and sums over a workgroup.  Included by .hip translation units only; everything has internal linkage.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "ivfpq_hip_util.hpp"

namespace {

constexpr float kLog2E = 1.44269504f, kLn2 = 0.69314718f;

typedef _Float16 half_t;
typedef __bf16 bf16_t;

inline int value_bytes(int dtype) { return dtype == IVFPQ_VALUES_FP32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == IVFPQ_VALUES_FP32 || dtype == IVFPQ_VALUES_FP16 || dtype == IVFPQ_VALUES_BF16; }

// Calls f with a value of the C++ type of `dtype` (one that known_dtype accepts).
template <class F>
int with_value_type(int dtype, F&& f) {
    if (dtype == IVFPQ_VALUES_FP16) return f(half_t{});
    if (dtype == IVFPQ_VALUES_BF16) return f(bf16_t{});
    return f(float{});
}

// VEC consecutive values, 16 bytes
template <class T>
struct Chunk {
    static constexpr int VEC = 16 / sizeof(T);
    uint4 bits;
    __device__ inline void widen(float (&x)[VEC]) const {
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
        } else if constexpr (std::is_same<T, bf16_t>::value) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                typedef half_t half2_t __attribute__((ext_vector_type(2)));
                const half2_t h = __builtin_bit_cast(half2_t, w[i]);
                x[2 * i] = (float)h.x;
                x[2 * i + 1] = (float)h.y;
            }
        }
    }
    // Keeps the compiler from holding the widened values of one use for the next: a tile of them does not fit the registers.
    __device__ inline void forget_widened() { asm volatile("" : "+v"(bits.x), "+v"(bits.y), "+v"(bits.z), "+v"(bits.w)); }
    // rounds to nearest, ties to even
    __device__ inline void narrow(const float (&x)[VEC]) {
        typedef T vec_t __attribute__((ext_vector_type(VEC)));
        vec_t v;
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (T)x[i];
        bits = __builtin_bit_cast(uint4, v);
    }
};

// A row seen as 16-byte chunks at 16-byte boundaries, whatever its own alignment: value v is element v + lead of the chunks.
// The first and the last chunk may lie partly outside of the row; those are read and written value by value.
template <class T>
struct RowChunks {
    static constexpr int VEC = Chunk<T>::VEC;
    const T* row;
    const uint4* base;
    int lead, end;                   // elements [lead, end) are the row's
    __device__ RowChunks(const void* data, long long r, long long stride, int count) {
        row = reinterpret_cast<const T*>(data) + r * stride;
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        base = reinterpret_cast<const uint4*>(row - lead);       // by pointer arithmetic, so that its loads are known to be of global memory
        end = lead + count;
    }
    __device__ inline int count() const { return (end + VEC - 1) / VEC; }
    // chunks [first_whole, end_whole) lie inside of the row; the one before and the one behind hold the rest of it
    __device__ inline int first_whole() const { return lead ? 1 : 0; }
    __device__ inline int end_whole() const { return end / VEC; }
    __device__ inline bool whole(int c) const { return c * VEC >= lead && (c + 1) * VEC <= end; }
    __device__ inline float value(int v) const { return (float)row[v]; }
    // `fill` stands for values outside of the row
    __device__ inline Chunk<T> load(int c, float fill = -INFINITY) const {
        Chunk<T> k;
        if (whole(c)) {
            k.bits = base[c];
            return k;
        }
        float x[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int e = c * VEC + i;
            x[i] = e >= lead && e < end ? (float)row[e - lead] : fill;
        }
        k.narrow(x);
        return k;
    }
};

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }       // results under 2^-126 are 0

// The largest of three; NaNs are passed over.  (fmaxf of values that come from integer operations costs a second instruction each, which
// makes quiet a signalling NaN.)
__device__ inline float max3(float a, float b, float c) {
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// The sum of N values, halves added up apart
template <int N>
__device__ inline float tree_sum(const float* x) {
    if constexpr (N == 1) return x[0];
    else return tree_sum<N / 2>(x) + tree_sum<N - N / 2>(x + N / 2);
}

// The sum over a workgroup of THREADS, in every thread; the order of additions is fixed.  `scratch`: THREADS / 64 words that no
// wave still reads; they are free again after the next barrier.
template <int THREADS, class V>
__device__ inline V block_sum(V x, V* scratch) {
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    V sum = scratch[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) sum += scratch[w];
    __syncthreads();
    return sum;
}
template <int THREADS>
__device__ inline float block_max(float x, float* scratch) {
    for (int off = 32; off; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    float most = scratch[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) most = fmaxf(most, scratch[w]);
    __syncthreads();
    return most;
}

}  // namespace
