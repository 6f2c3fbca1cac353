// The 8-bit form of a block of 128 elements: its scale from the largest magnitude, its codes.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace mw {

constexpr uint8_t kFp8NanScale = 0xff;

// A magnitude's bits, which order as the magnitudes do, infinities and NaN above.
__device__ __forceinline__ uint32_t fp8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The largest magnitude of three, NaN where one is (one instruction).
__device__ __forceinline__ float fp8_largest(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// The exponent byte of the least power of two s with top <= 448 s: 448 = 1.75 x 2^8, so the
// exponent is top's less 8, or less 7 for a fraction over 1.75 (the sum carries into it).
__device__ __forceinline__ uint8_t fp8_scale(uint32_t top) {
  const int e = static_cast<int>((top + 0x1fffffu) >> 23) - 8;
  return top >= 0x7f800000u ? kFp8NanScale : static_cast<uint8_t>(max(e, 0));
}

// The same of the two bf16 magnitudes of a word, in its halves.
__device__ __forceinline__ uint32_t fp8_scale2(uint32_t tops) {
  const uint32_t e = __vmaxu2(((tops + 0x001f001fu) >> 7) & 0x00ff00ffu, 0x00080008u) - 0x00080008u;
  const uint32_t over = (tops + 0x00800080u) & 0x80008000u;  // not finite
  return e | ((over >> 7) - (over >> 15));
}

// 1 / s (NaN for NaN): 7 <= 254 - scale <= 254, a normal number.
__device__ __forceinline__ float fp8_inverse(uint8_t scale) {
  return __uint_as_float(scale == kFp8NanScale ? 0x7fffffffu : (254u - scale) << 23);
}

// Two codes, a in the low byte.
__device__ __forceinline__ uint32_t fp8_pair(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}

// Four codes.
__device__ __forceinline__ uint32_t fp8_four(float2 a, float2 b) {
  return fp8_pair(a.x, a.y) | fp8_pair(b.x, b.y) << 16;
}

// Eight codes of values already divided by the scale (NaN where that is NaN).
__device__ __forceinline__ uint2 fp8_codes(const float (&v)[8]) {
  return make_uint2(fp8_four(make_float2(v[0], v[1]), make_float2(v[2], v[3])),
                    fp8_four(make_float2(v[4], v[5]), make_float2(v[6], v[7])));
}

}  // namespace mw
