// Activations into 8 bits and back: streaming kernels bound by HBM bandwidth
// (bf16: 2 bytes read or written and 1 + 1/32 the other way an element).
#include "ckpt8.h"

#include "kernels.h"

namespace strata {
namespace ckpt8 {

constexpr int kThreads = 256, kHalf = 8 * kThreads, kSpan = 2 * kHalf;

// One thread's 8 elements at `at`, any n: the last block's.
template <bool BF16>
__device__ __forceinline__ void pack_part(const void* x, int64_t at, int64_t n, int8_t* codes, uint8_t* scales) {
  Raw8<BF16> raw;
  raw.load_part(x, at, n);
  float v[8];
  raw.get(v);
  const uint32_t e = exponent_of(group_top(raw));
  const uint2 c = encode8(v, e);
  if (at < n && (threadIdx.x & 3) == 0) scales[at >> 5] = (uint8_t)e;
  const uint64_t w = (uint64_t)c.y << 32 | c.x;
  for (int j = 0; j < 8 && at + j < n; ++j) codes[at + j] = (int8_t)(w >> (8 * j));
}

// A block takes two runs of 2048 elements, a thread 8 of each; neighbouring lanes
// swap half of their codes, so that each stores 16 bytes of one run, and 16 lanes
// gather their 4 exponents into a word.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) pack_kernel(const void* __restrict__ x, int64_t n,
                                                        int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t base = block_index() * kSpan, at = base + 8 * threadIdx.x;
  if (base + kSpan > n) {
    pack_part<BF16>(x, at, n, codes, scales);
    pack_part<BF16>(x, at + kHalf, n, codes, scales);
    return;
  }
  constexpr int kBytes = BF16 ? 2 : 4;
  Raw8<BF16> raw[2];
  raw[0].template load<true>(static_cast<const char*>(x) + at * kBytes);
  raw[1].template load<true>(static_cast<const char*>(x) + (at + kHalf) * kBytes);
  uint2 c[2];
  uint32_t e[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    raw[i].get(v);
    e[i] = exponent_of(group_top(raw[i]));
    c[i] = encode8(v, e[i]);
    e[i] = quads_or<16>(e[i] << (8 * (threadIdx.x >> 2 & 3)));
  }
  const int odd = threadIdx.x & 1;
  swap_pair(odd, c[0], c[1]);
  store16(codes + at + (odd ? kHalf - 8 : 0), u32x4{c[0].x, c[0].y, c[1].x, c[1].y});
  if ((threadIdx.x & 15) < 2)
    *reinterpret_cast<uint32_t*>(scales + ((at - 8 * odd + odd * kHalf) >> 5)) = odd ? e[1] : e[0];
}

template <bool BF16>
__device__ __forceinline__ void unpack_part(const int8_t* codes, const uint8_t* scales, int64_t at, int64_t n, void* x) {
  if (at >= n) return;
  const float step = step_of(scales[at >> 5]);
  for (int j = 0; j < 8 && at + j < n; ++j) store1<BF16>(x, at + j, (float)codes[at + j] * step);
}

// The same the other way.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const int8_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales, int64_t n,
                                                          void* __restrict__ x) {
  const int64_t base = block_index() * kSpan, at = base + 8 * threadIdx.x;
  if (base + kSpan > n) {
    unpack_part<BF16>(codes, scales, at, n, x);
    unpack_part<BF16>(codes, scales, at + kHalf, n, x);
    return;
  }
  constexpr int kBytes = BF16 ? 2 : 4;
  const int odd = threadIdx.x & 1;
  const u32x4 w = load16(codes + at + (odd ? kHalf - 8 : 0));
  const uint8_t e[2] = {scales[at >> 5], scales[(at + kHalf) >> 5]};
  uint2 c[2] = {make_uint2(w.x, w.y), make_uint2(w.z, w.w)};
  swap_pair(odd, c[0], c[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    decode8(c[i], step_of(e[i]), v);
    store8_stream<BF16>(static_cast<char*>(x) + (at + i * kHalf) * kBytes, v);
  }
}

static dim3 blocks_for(int64_t n) { return grid_of((n + kSpan - 1) / kSpan); }

}  // namespace ckpt8

void launch_ckpt_pack(const void* x, int64_t n, int8_t* codes, uint8_t* scales, strata_dtype dt, hipStream_t s) {
  const dim3 grid = ckpt8::blocks_for(n);
  if (dt == STRATA_BF16)
    hipLaunchKernelGGL(ckpt8::pack_kernel<true>, grid, dim3(ckpt8::kThreads), 0, s, x, n, codes, scales);
  else
    hipLaunchKernelGGL(ckpt8::pack_kernel<false>, grid, dim3(ckpt8::kThreads), 0, s, x, n, codes, scales);
}

void launch_ckpt_unpack(const int8_t* codes, const uint8_t* scales, int64_t n, void* x, strata_dtype dt,
                        hipStream_t s) {
  const dim3 grid = ckpt8::blocks_for(n);
  if (dt == STRATA_BF16)
    hipLaunchKernelGGL(ckpt8::unpack_kernel<true>, grid, dim3(ckpt8::kThreads), 0, s, codes, scales, n, x);
  else
    hipLaunchKernelGGL(ckpt8::unpack_kernel<false>, grid, dim3(ckpt8::kThreads), 0, s, codes, scales, n, x);
}

}  // namespace strata
