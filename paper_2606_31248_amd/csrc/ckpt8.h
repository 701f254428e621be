// The 8-bit form of activations: groups of 32 consecutive elements as int8 codes
// times a power of two.  A lane holds 8 elements, a quad of lanes one group.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "mfma_util.h"

namespace strata {
namespace ckpt8 {

constexpr int kGroup = 32;

// lanes of a DPP row exchanged without LDS: quad_perm [1,0,3,2], [2,3,0,1], the
// mirror of 8 lanes and of 16
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, false);
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes that are touched once: past the caches' replacement, which leaves them to
// what is read again
__device__ __forceinline__ u32x4 load16(const void* p) {
  return __builtin_nontemporal_load(static_cast<const u32x4*>(p));
}
__device__ __forceinline__ void store16(void* p, u32x4 v) { __builtin_nontemporal_store(v, static_cast<u32x4*>(p)); }

__device__ __forceinline__ void widen(u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = mfma::lo_bf16(r[i]), v[2 * i + 1] = mfma::hi_bf16(r[i]);
}
__device__ __forceinline__ void as_floats(u32x4 a, u32x4 b, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
}

// 8 elements as they lie in memory: 16 bytes of bf16 or 32 of float32.  STREAM: past
// the caches' replacement; bf16 alone, since the two halves of a lane's float32 meet in
// the same cache lines.
template <bool BF16>
struct Raw8;
template <>
struct Raw8<true> {
  u32x4 a;
  template <bool STREAM>
  __device__ __forceinline__ void load(const void* p) {
    a = STREAM ? load16(p) : *static_cast<const u32x4*>(p);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { widen(a, v); }
  // elements [at, n) of less than 8, then zeros
  __device__ __forceinline__ void load_part(const void* p, int64_t at, int64_t n) {
    const uint16_t* q = static_cast<const uint16_t*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      a[j] = (at + 2 * j < n ? q[at + 2 * j] : 0u) | (at + 2 * j + 1 < n ? (uint32_t)q[at + 2 * j + 1] << 16 : 0u);
  }
};
template <>
struct Raw8<false> {
  u32x4 a, b;
  template <bool STREAM>
  __device__ __forceinline__ void load(const void* p) {
    a = static_cast<const u32x4*>(p)[0], b = static_cast<const u32x4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { as_floats(a, b, v); }
  __device__ __forceinline__ void load_part(const void* p, int64_t at, int64_t n) {
    const uint32_t* q = static_cast<const uint32_t*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = at + j < n ? q[at + j] : 0u, b[j] = at + 4 + j < n ? q[at + 4 + j] : 0u;
  }
};

// past the caches' replacement in bf16 (float32: its two halves meet in the caches)
template <bool BF16>
__device__ __forceinline__ void store8_stream(void* p, const float (&v)[8]) {
  if (BF16) {
    store16(p, u32x4{mfma::pack2(v[0], v[1]), mfma::pack2(v[2], v[3]), mfma::pack2(v[4], v[5]), mfma::pack2(v[6], v[7])});
  } else {
    u32x4* q = static_cast<u32x4*>(p);
    q[0] = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    q[1] = u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
  }
}

template <bool BF16>
__device__ __forceinline__ void store1(void* p, int64_t at, float v) {
  if (BF16)
    static_cast<uint16_t*>(p)[at] = f32_to_bf16(v);
  else
    static_cast<float*>(p)[at] = v;
}

// Block index in a two-dimensional grid: HIP wants gridDim.x * blockDim.x below
// 2^32, and a card's largest activations exceed that.
__device__ __forceinline__ int64_t block_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

inline dim3 grid_of(int64_t blocks) {
  const int64_t y = (blocks + (1 << 20) - 1) >> 20;
  return dim3((unsigned)((blocks + y - 1) / y), (unsigned)y);
}

// Biased exponent of the group whose largest |bits| is `top`: where 2^(E - 133)
// would make it round to 128 steps (mantissa >= 127.5/64) the sum carries into the
// exponent.  255: an infinity or a NaN among the 32.
__device__ __forceinline__ uint32_t exponent_of(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const uint32_t e = (top + 0x10000u) >> 23;
  return e < 7u ? 7u : (e > 254u ? 254u : e);
}

// 2^(E - 133), normal for every E in [7, 254]; NaN for 255, so that the group decodes as NaN
__device__ __forceinline__ float step_of(uint32_t e) {
  return __uint_as_float(e == 255u ? 0x7FC00000u : (e - 6u) << 23);
}

// Codes of 8 values (4 bytes a word): v 2^(133 - E), exact, plus 1.5 * 2^23 in one
// fused multiply-add rounds to an integer, ties to even, whose two's complement is
// the sum's low byte.  Only E = 254 can round to 128.
__device__ __forceinline__ uint2 encode8(const float (&v)[8], uint32_t e) {
  constexpr float kRound = 12582912.f;
  const float inv = __uint_as_float((260u - e) << 23);
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(v[i], inv, kRound));
  if (e >= 254u) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      b[i] = e == 255u ? 0u : __float_as_uint(__builtin_amdgcn_fmed3f(v[i] * inv, -127.f, 127.f) + kRound);
  }
  auto pack = [](uint32_t p, uint32_t q, uint32_t r, uint32_t s) {  // the low byte of each
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(s, r, 0x0C0C0400u), __builtin_amdgcn_perm(q, p, 0x0C0C0400u),
                                 0x05040100u);
  };
  return make_uint2(pack(b[0], b[1], b[2], b[3]), pack(b[4], b[5], b[6], b[7]));
}

// code + 128 of the i-th of 8 codes whose words were flipped by 0x80808080: unsigned
// bytes convert in one instruction
__device__ __forceinline__ float code_up(uint2 flipped, int i) {
  return (float)(((i < 4 ? flipped.x : flipped.y) >> (8 * (i & 3))) & 255u);
}
__device__ __forceinline__ uint2 flip(uint2 c) { return make_uint2(c.x ^ 0x80808080u, c.y ^ 0x80808080u); }

// 8 codes -> values
__device__ __forceinline__ void decode8(uint2 c, float step, float (&v)[8]) {
  const uint2 w = flip(c);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (code_up(w, i) - 128.f) * step;
}

// 8 codes -> values times f, rounded once: (code + 128) F - 128 F with F = step f.
// F has to stay below 2^120 (a step of 2^121 only with f = 0); as a subnormal it is
// itself rounded.
__device__ __forceinline__ void decode8_times(uint2 c, float step, float f, float (&v)[8]) {
  const uint2 w = flip(c);
  const float m = step * f, off = -128.f * m;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(code_up(w, i), m, off);
}

// Sum of the squares of 8 codes, below 2^17 and so exact, as the sum of their values'
// squares over step^2 is in float32 where those are normal numbers
__device__ __forceinline__ float code_squares(uint2 c) {
  return (float)__builtin_amdgcn_sdot4((int)c.x, (int)c.x, __builtin_amdgcn_sdot4((int)c.y, (int)c.y, 0, false), false);
}

// OR over the quads of LANES neighbouring lanes
template <int LANES>
__device__ __forceinline__ uint32_t quads_or(uint32_t x) {
  if (LANES >= 8) x |= dpp<kMirror8>(x);
  if (LANES >= 16) x |= dpp<kMirror16>(x);
  return x;
}

// Two neighbouring slices' codes between "each lane its 8 of both" and "an even lane 16 of
// the first slice, its own and the next lane's, an odd lane 16 of the second"; its own inverse.
__device__ __forceinline__ void swap_pair(int odd, uint2& first, uint2& second) {
  const uint32_t gx = dpp<kSwap1>(odd ? first.x : second.x), gy = dpp<kSwap1>(odd ? first.y : second.y);
  (odd ? first : second) = make_uint2(gx, gy);
}

// largest |bits|, as float32, of the quad's 32 values: bf16 as they lie, two to a word
__device__ __forceinline__ uint32_t group_top(const Raw8<true>& raw) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto half = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(half(raw.a[0]), half(raw.a[1])),
                                            __builtin_elementwise_max(half(raw.a[2]), half(raw.a[3])));
  uint32_t t = (uint32_t)(m.x > m.y ? m.x : m.y) << 16;
  t = umax(t, dpp<kSwap1>(t));
  return umax(t, dpp<kSwap2>(t));
}

__device__ __forceinline__ uint32_t group_top(const Raw8<false>& raw) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t = umax(t, umax(raw.a[i] & 0x7FFFFFFFu, raw.b[i] & 0x7FFFFFFFu));
  t = umax(t, dpp<kSwap1>(t));
  return umax(t, dpp<kSwap2>(t));
}

}  // namespace ckpt8
}  // namespace strata
