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

// 8 elements as they lie in memory: 16 bytes of bf16 or 32 of float32
template <bool BF16>
struct Raw8;
template <>
struct Raw8<true> {
  u32x4 a;
  __device__ __forceinline__ void load(const void* p) { a = load16(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const { widen(a, v); }
};
template <>
struct Raw8<false> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const void* p) { a = load16(p), b = load16(static_cast<const char*>(p) + 16); }
  __device__ __forceinline__ void get(float (&v)[8]) const { as_floats(a, b, v); }
};

template <bool BF16>
__device__ __forceinline__ void store8_stream(void* p, const float (&v)[8]) {
  if (BF16) {
    store16(p, u32x4{mfma::pack2(v[0], v[1]), mfma::pack2(v[2], v[3]), mfma::pack2(v[4], v[5]), mfma::pack2(v[6], v[7])});
  } else {
    store16(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    store16(static_cast<char*>(p) + 16,
            u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
  }
}

template <bool BF16>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
  return BF16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[at]) : static_cast<const float*>(p)[at];
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

// Codes of 8 values (4 bytes a word) with the inverse step 2^(133 - E): the
// product is exact, and adding 1.5 * 2^23 rounds it to an integer, ties to even,
// whose two's complement is the sum's low byte.
__device__ __forceinline__ uint2 encode8(const float (&v)[8], uint32_t e) {
  if (e == 255u) return make_uint2(0u, 0u);
  const float inv = __uint_as_float((260u - e) << 23);
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    b[i] = __float_as_uint(__builtin_amdgcn_fmed3f(v[i] * inv, -127.f, 127.f) + 12582912.f);
  auto pack = [](uint32_t p, uint32_t q, uint32_t r, uint32_t s) {
    return (p & 255u) | (q & 255u) << 8 | (r & 255u) << 16 | s << 24;
  };
  return make_uint2(pack(b[0], b[1], b[2], b[3]), pack(b[4], b[5], b[6], b[7]));
}

// 8 codes -> values
__device__ __forceinline__ void decode8(uint2 c, float step, float (&v)[8]) {
  const uint32_t w[2] = {c.x ^ 0x80808080u, c.y ^ 0x80808080u};  // code + 128: unsigned bytes convert in one instruction
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = ((float)((w[i >> 2] >> (8 * (i & 3))) & 255u) - 128.f) * step;
}

// Two neighbouring slices' codes between "each lane its 8 of both" and "an even lane 16 of
// the first slice, its own and the next lane's, an odd lane 16 of the second"; its own inverse.
__device__ __forceinline__ void swap_pair(int odd, uint2& first, uint2& second) {
  const uint32_t gx = dpp<kSwap1>(odd ? first.x : second.x), gy = dpp<kSwap1>(odd ? first.y : second.y);
  (odd ? first : second) = make_uint2(gx, gy);
}

// largest |bits| of the quad's 32 values
__device__ __forceinline__ uint32_t group_top(const float (&v)[8]) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = umax(t, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  t = umax(t, dpp<kSwap1>(t));
  return umax(t, dpp<kSwap2>(t));
}

}  // namespace ckpt8
}  // namespace strata
