// AdamW over many tensors at once, the 8-bit form of its states, and the norm of all gradients.
//
// Every element is read and written once: 28 bytes with states in 32 bits, bf16 gradients
// and a bf16 copy, 16 with states in 8.  HBM bounds the first (15 operations an element),
// the second has about 60 operations beside it.  A block takes kParamChunk elements of one
// tensor; a lane 4 neighbouring ones at a time, 16 bytes of float32, so that 8 lanes hold a
// group of the 8-bit states.
#include "state8.h"

#include "kernels.h"

namespace strata {
namespace adamw {

using namespace ckpt8;

constexpr int kThreads = 256, kSpan = 4 * kThreads, kParts = kParamChunk / kSpan;

// A lane's 4 gradients, n of them there.
__device__ __forceinline__ void load_grads(const ParamRecord& t, int64_t at, int n, float (&g)[4]) {
  if (t.bf16) {
    const uint16_t* q = static_cast<const uint16_t*>(t.g) + at;
    if (n == 4) {
      const uint2 w = *reinterpret_cast<const uint2*>(q);
      g[0] = mfma::lo_bf16(w.x), g[1] = mfma::hi_bf16(w.x), g[2] = mfma::lo_bf16(w.y), g[3] = mfma::hi_bf16(w.y);
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = j < n ? bf16_to_f32(q[j]) : 0.f;
  } else {
    const float* q = static_cast<const float*>(t.g) + at;
    if (n == 4) {
      const float4 w = *reinterpret_cast<const float4*>(q);
      g[0] = w.x, g[1] = w.y, g[2] = w.z, g[3] = w.w;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = j < n ? q[j] : 0.f;
  }
}

__device__ __forceinline__ void load_floats(const float* q, int n, float (&v)[4]) {
  if (n == 4) {
    const float4 w = *reinterpret_cast<const float4*>(q);
    v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = j < n ? q[j] : 0.f;
}

__device__ __forceinline__ void store_floats(float* q, int n, const float (&v)[4]) {
  if (n == 4) {
    *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) q[j] = v[j];
}

__device__ __forceinline__ void store_copy(uint16_t* q, int n, const float (&v)[4]) {
  if (n == 4) {
    *reinterpret_cast<uint2*>(q) = make_uint2(mfma::pack2(v[0], v[1]), mfma::pack2(v[2], v[3]));
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) q[j] = f32_to_bf16(v[j]);
}

// The group's largest |bits| in each of its 8 lanes.
__device__ __forceinline__ uint32_t group_top(const float (&v)[4]) {
  uint32_t t = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) t = umax(t, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  t = umax(t, dpp<kSwap1>(t));
  t = umax(t, dpp<kSwap2>(t));
  return umax(t, dpp<kMirror8>(t));
}

// A lane's 4 values of a state, decoded, and encoded again.
template <bool SECOND>
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t e, float (&v)[4]) {
  const float unit = state8::unit_of<SECOND>(e);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = state8::decode<SECOND>(codes >> (8 * j) & 255u, unit);
}

template <bool SECOND>
__device__ __forceinline__ void store4(void* codes, uint8_t* scales, int64_t place, const float (&v)[4],
                                       const uint32_t (&random)[4]) {
  const uint32_t e = state8::exponent_of<SECOND>(group_top(v));
  uint32_t w = 0;
  if (e != 255u) {
    const float per_unit = state8::per_unit_of<SECOND>(e);
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= state8::encode<SECOND>(v[j], per_unit, random[j]) << (8 * j);
  }
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(codes) + place) = w;
  if ((threadIdx.x & 7) == 0) scales[place >> 5] = (uint8_t)e;
}

template <bool EIGHT>
__global__ void __launch_bounds__(kThreads) step_kernel(const AdamArgs a) {
  const int64_t chunk = block_index();
  if (chunk >= a.chunks) return;
  const float factor = a.factor ? *a.factor : 1.f;
  if (factor != factor) return;  // gradients that are not finite: nothing changes
  const ParamRecord t = a.tensors[a.owner[chunk]];
  const int64_t first = (chunk - t.chunk) * kParamChunk + 4 * threadIdx.x;
  float p[kParts][4], g[kParts][4], m[kParts][4], v[kParts][4];
  uint32_t mc[kParts], vc[kParts], me[kParts], ve[kParts];
  int n[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const int64_t at = first + i * kSpan, left = t.n - at, place = t.place + at;
    n[i] = left >= 4 ? 4 : left > 0 ? (int)left : 0;
    if (EIGHT ? t.n <= (at & -32) : n[i] == 0) {  // lanes of a group stay together
      n[i] = -1;
      continue;
    }
    load_grads(t, at, n[i], g[i]);
    load_floats(t.p + at, n[i], p[i]);
    if (EIGHT) {
      mc[i] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.m) + place);
      vc[i] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.v) + place);
      me[i] = a.m_scales[place >> 5], ve[i] = a.v_scales[place >> 5];
    } else {
      load_floats(static_cast<const float*>(a.m) + place, n[i], m[i]);
      load_floats(static_cast<const float*>(a.v) + place, n[i], v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    if (n[i] < 0) continue;
    const int64_t at = first + i * kSpan, place = t.place + at;
    if (EIGHT) decode4<false>(mc[i], me[i], m[i]), decode4<true>(vc[i], ve[i], v[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // each product and sum rounded by itself, so that the states do not hang on how they were fused
#pragma clang fp contract(off)
      const float x = g[i][j] * factor;
      m[i][j] = a.beta1 * m[i][j] + a.new1 * x;
      v[i][j] = a.beta2 * v[i][j] + a.new2 * x * x;
      if (EIGHT && j >= n[i]) m[i][j] = v[i][j] = 0.f;
      const float root = sqrtf(v[i][j]) * a.root + a.eps;
      p[i][j] = p[i][j] - (a.decay * p[i][j] + a.rate * m[i][j] / root);
    }
    store_floats(t.p + at, n[i], p[i]);
    if (t.copy) store_copy(t.copy + at, n[i], p[i]);
    if (EIGHT) {
      uint32_t low[4], high[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t r = state8::mix((uint32_t)(place + j) ^ a.key);
        low[j] = r & 0xFFFFu, high[j] = r >> 16;
      }
      store4<false>(a.m, a.m_scales, place, m[i], low);
      store4<true>(a.v, a.v_scales, place, v[i], high);
    } else {
      store_floats(static_cast<float*>(a.m) + place, n[i], m[i]);
      store_floats(static_cast<float*>(a.v) + place, n[i], v[i]);
    }
  }
}

// Values of a state: a lane 8 codes, any n.
template <bool BF16, bool SECOND>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const uint8_t* codes, const uint8_t* scales, int64_t n, void* x) {
  const int64_t at = (block_index() * kThreads + threadIdx.x) * 8;
  if (at >= n) return;
  const float unit = state8::unit_of<SECOND>(scales[at >> 5]);
  if (at + 8 <= n) {
    const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = state8::decode<SECOND>((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255u, unit);
    store8_stream<BF16>(static_cast<char*>(x) + at * (BF16 ? 2 : 4), v);
    return;
  }
  for (int j = 0; at + j < n; ++j) store1<BF16>(x, at + j, state8::decode<SECOND>(codes[at + j], unit));
}

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double sums[kThreads];
  sums[threadIdx.x] = x;
  __syncthreads();
#pragma unroll
  for (int d = kThreads / 2; d > 0; d /= 2) {
    if (threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
    __syncthreads();
  }
  return sums[0];
}

// Squares of float32 values in float64: neither range nor digits are lost, whatever the count.
__global__ void __launch_bounds__(kThreads) squares_kernel(const ParamRecord* tensors, const int32_t* owner,
                                                           int64_t chunks, double* partial) {
  double x = 0.;
  for (int64_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    const ParamRecord t = tensors[owner[chunk]];
    const int64_t first = (chunk - t.chunk) * kParamChunk + 4 * threadIdx.x;
    float g[kParts][4];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int64_t at = first + i * kSpan, left = t.n - at;
      load_grads(t, at, left >= 4 ? 4 : left > 0 ? (int)left : 0, g[i]);
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x = fma((double)g[i][j], (double)g[i][j], x);
  }
  x = block_sum(x);
  if (threadIdx.x == 0) partial[blockIdx.x] = x;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* partial, int blocks, double most, float* norm) {
  double x = 0.;
  for (int i = threadIdx.x; i < blocks; i += kThreads) x += partial[i];
  x = sqrt(block_sum(x));
  if (threadIdx.x) return;
  norm[0] = (float)x;
  norm[1] = !(x <= 0x1.fffffffffffffp1023) ? __uint_as_float(0x7FC00000u) : x <= most ? 1.f : (float)(most / x);
}

constexpr int kNormBlocks = 2048;

}  // namespace adamw

uint32_t adamw_key(uint64_t seed) {
  return state8::mix(state8::mix((uint32_t)seed + 0x3C6EF372u) ^ (uint32_t)(seed >> 32));
}

void launch_adamw(const AdamArgs& a, hipStream_t s) {
  const dim3 grid = ckpt8::grid_of(a.chunks), block(adamw::kThreads);
  if (a.m_scales)
    hipLaunchKernelGGL(adamw::step_kernel<true>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(adamw::step_kernel<false>, grid, block, 0, s, a);
}

void launch_adamw_unpack(const uint8_t* codes, const uint8_t* scales, int64_t n, bool second, void* x, strata_dtype dt,
                         hipStream_t s) {
  const dim3 grid = ckpt8::grid_of((n + 8 * adamw::kThreads - 1) / (8 * adamw::kThreads)), block(adamw::kThreads);
  if (dt == STRATA_BF16) {
    if (second)
      hipLaunchKernelGGL((adamw::unpack_kernel<true, true>), grid, block, 0, s, codes, scales, n, x);
    else
      hipLaunchKernelGGL((adamw::unpack_kernel<true, false>), grid, block, 0, s, codes, scales, n, x);
  } else if (second) {
    hipLaunchKernelGGL((adamw::unpack_kernel<false, true>), grid, block, 0, s, codes, scales, n, x);
  } else {
    hipLaunchKernelGGL((adamw::unpack_kernel<false, false>), grid, block, 0, s, codes, scales, n, x);
  }
}

int64_t grad_norm_blocks(int64_t chunks) { return chunks < adamw::kNormBlocks ? chunks : adamw::kNormBlocks; }

void launch_grad_norm(const ParamRecord* tensors, const int32_t* owner, int64_t chunks, double most, float* norm,
                      double* partial, hipStream_t s) {
  const int blocks = (int)grad_norm_blocks(chunks);
  if (blocks)
    hipLaunchKernelGGL(adamw::squares_kernel, dim3(blocks), dim3(adamw::kThreads), 0, s, tensors, owner, chunks, partial);
  hipLaunchKernelGGL(adamw::norm_kernel, dim3(1), dim3(adamw::kThreads), 0, s, partial, blocks, most, norm);
}

}  // namespace strata
