// The optimiser's states in 8 bits: groups of 32 consecutive values with an exponent.
// A first moment has a sign, 4 bits of exponent and 3 behind the leading one, a second
// moment, never negative, 5 and 3: moments of one group lie many octaves apart, and the
// square root halves the second's distance.  With E the biased exponent of the group's
// largest value (one more where it would round to 16 eighths), the unit is
// 2^(E - 127 - kUnit); code c stands for c units below 8 and for
// (8 + c mod 8) 2^(c div 8 - 1) units above, which are the bits of a float.
#pragma once

#include "ckpt8.h"

namespace strata {
namespace state8 {

using namespace ckpt8;

template <bool SECOND>
struct Form {
  static constexpr int kUnit = SECOND ? 33 : 17;  // octaves from the exponent of the largest to the unit
};

// From the largest |bits| of the group.  At least kUnit + 1, so that the unit is a normal
// number; 255: an infinity or a NaN among the 32.
template <bool SECOND>
__device__ __forceinline__ uint32_t exponent_of(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const uint32_t e = (top + 0x100000u) >> 23, least = Form<SECOND>::kUnit + 1;
  return e < least ? least : e > 254u ? 254u : e;
}

// One unit, and its reciprocal.  Of states that start as zeros the exponents are 0; NaN for 255.
template <bool SECOND>
__device__ __forceinline__ float unit_of(uint32_t e) {
  const int u = (int)e - Form<SECOND>::kUnit;
  return __uint_as_float(e == 255u ? 0x7FC00000u : (uint32_t)(u < 1 ? 1 : u) << 23);
}
template <bool SECOND>
__device__ __forceinline__ float per_unit_of(uint32_t e) {
  return __uint_as_float((254u + Form<SECOND>::kUnit - e) << 23);
}

// Codes 8 and more are the top bits of a float between 8 and 2^kUnit, less these.
constexpr uint32_t kBits = 1032u;  // of 8 = 2^3: (127 + 3) << 3, less the code 8

template <bool SECOND>
__device__ __forceinline__ float decode(uint32_t byte, float unit) {
  const uint32_t c = SECOND ? byte : byte & 127u;
  const float low = (float)c, high = __uint_as_float((c + kBits) << 20);
  const float v = (c < 8u ? low : high) * unit;
  return SECOND ? v : __uint_as_float(__float_as_uint(v) | (byte & 128u) << 24);
}

// Rounded up where `random`, 16 bits, reaches over the border: the mean over the random
// numbers is x.  A second moment above 0 keeps code 1: it is divided by.  Without branches:
// the code of the part below 8 and that of the part above, one of which is 8.  Only at the
// largest scale, which cannot be one more, is there a code too many.
template <bool SECOND>
__device__ __forceinline__ uint32_t encode(float x, float per_unit, uint32_t random) {
  const float t = fabsf(x) * per_unit;
  const uint32_t low = (uint32_t)(fminf(t, 8.f) + (float)random * 0x1p-16f);
  const uint32_t high = (__float_as_uint(fmaxf(t, 8.f)) + (random << 4)) >> 20;
  const uint32_t c = low + high - (kBits + 8u);
  if (SECOND) return min(umax(c, x > 0.f ? 1u : 0u), 255u);
  return min(c, 127u) | (__float_as_uint(x) >> 24 & 128u);
}

// 32 bits of (seed, element): two rounds of a product and a shift, which move every bit.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ x >> 16) * 0x6A09E667u;
  x = (x ^ x >> 15) * 0xBB67AE85u;
  return x ^ x >> 16;
}

}  // namespace state8
}  // namespace strata
