// The power-of-two scales of an 8-bit cache, for the kernels that choose them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dv {

// The smallest power of two, at least 2^-64, whose 448-fold is at least amax
// (448 = 1.75 * 2^8): from amax's exponent, one more where its fraction exceeds
// 1.75.
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) + ((b & 0x7fffff) > 0x600000) - 8;
  return __uint_as_float((uint32_t)max(e, 127 - 64) << 23);
}

// 1 / p for a power of two of [2^-64, 2^120].
__device__ __forceinline__ float inverse(float p) {
  return __uint_as_float((254u << 23) - __float_as_uint(p));
}

}  // namespace dv
