// Order-preserving unsigned keys of floats.  Included by .hip translation units only; everything has internal linkage.
#pragma once

#include <hip/hip_runtime.h>

namespace {

__device__ inline uint32_t ordered_key(float f) {          // monotone map float -> uint32
    const uint32_t b = __float_as_uint(f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ inline float ordered_key_value(uint32_t key) {
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}

}  // namespace
