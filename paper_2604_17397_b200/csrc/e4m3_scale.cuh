// Power-of-two scales of E4M3 blocks.
#pragma once

#include <stdint.h>

namespace sdvg {

// The smallest e in [-126, 120] with largest <= 448 * 2^e (448 = 1.75 * 2^8); `largest` is the bit pattern of a float that is >= 0 or
// +inf, never NaN.  A subnormal has exponent field 0 and falls below the range, as zero does; infinity has 255 and gives 120.
__device__ __forceinline__ int scale_exponent(uint32_t largest) {
  const int e = (int)(largest >> 23) - 135 + ((largest & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, -126), 120);
}
// The larger of a largest magnitude so far (0 at first) and |v|; a NaN, which sets no scale, is dropped.
__device__ __forceinline__ float larger(float top, float v) { return fmaxf(top, fabsf(v)); }
__device__ __forceinline__ float larger(float top, float a, float b) {
  float r;
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ int scale_exponent(float largest) { return scale_exponent(__float_as_uint(largest)); }
// Over the warp: magnitudes compare as their bits do.
__device__ __forceinline__ float warp_largest(float top) {
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((127 + e) << 23); }   // e in [-126, 127]
// The scale that an exponent byte stands for: 2^(byte - 127), NaN for 255.  Byte 0 is the subnormal 2^-127.
__device__ __forceinline__ float scale_of_byte(uint8_t b) {
  return __int_as_float(b == 0 ? 0x00400000 : b == 255 ? 0x7fffffff : (int)b << 23);
}

}  // namespace sdvg
