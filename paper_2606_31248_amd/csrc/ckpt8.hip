// Activations into 8 bits and back: streaming kernels bound by HBM bandwidth
// (bf16: 2 bytes read or written and 1 + 1/32 the other way an element).
#include "ckpt8.h"

#include "kernels.h"

namespace strata {
namespace ckpt8 {

constexpr int kThreads = 256;

// One thread per 8 elements, the last thread element by element.  `full`: n / 8.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) pack_kernel(const void* __restrict__ x, int64_t n,
                                                        int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int64_t i = block_index() * kThreads + threadIdx.x;
  const int64_t at = i * 8;
  float v[8];
  if (at + 8 <= n) {
    Raw8<BF16> raw;
    raw.load(static_cast<const char*>(x) + at * (BF16 ? 2 : 4));
    raw.get(v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = at + j < n ? load1<BF16>(x, at + j) : 0.f;
  }
  const uint32_t e = exponent_of(group_top(v));
  const uint2 c = encode8(v, e);
  if (at >= n) return;
  if ((i & 3) == 0) scales[i >> 2] = (uint8_t)e;
  if (at + 8 <= n) {
    *reinterpret_cast<uint2*>(codes + at) = c;
  } else {
    const uint64_t w = (uint64_t)c.y << 32 | c.x;
    for (int j = 0; at + j < n; ++j) codes[at + j] = (int8_t)(w >> (8 * j));
  }
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const int8_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales, int64_t n,
                                                          void* __restrict__ x) {
  const int64_t i = block_index() * kThreads + threadIdx.x;
  const int64_t at = i * 8;
  if (at >= n) return;
  const float step = step_of(scales[i >> 2]);
  float v[8];
  if (at + 8 <= n) {
    decode8(*reinterpret_cast<const uint2*>(codes + at), step, v);
    store8_stream<BF16>(static_cast<char*>(x) + at * (BF16 ? 2 : 4), v);
  } else {
    for (int j = 0; at + j < n; ++j) store1<BF16>(x, at + j, (float)codes[at + j] * step);
  }
}

static dim3 blocks_for(int64_t n) { return grid_of((n + 8 * kThreads - 1) / (8 * kThreads)); }

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
