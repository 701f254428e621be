// AdamW over many tensors at once, the 8-bit form of its states, and the norm of all gradients.
//
// Every element is read and written once: 28 bytes with states in 32 bits, bf16 gradients
// and a bf16 copy, 16 with states in 8.  HBM bounds the first (all weights of 24 blocks of
// 1024 channels: 1525 us, 6.0 TB/s of 6.5 that a copy reaches); the second takes 83 vector
// instructions an element beside it, two thirds of its time (873 us, 6.0 TB/s).  A block takes kParamChunk elements of one
// tensor; a lane 4 neighbouring ones at a time, 16 bytes of float32, so that 8 lanes hold a
// group of the 8-bit states.
#include "state8.h"

#include "kernels.h"

namespace strata {
namespace adamw {

using namespace ckpt8;

constexpr int kThreads = 256, kSpan = 4 * kThreads;

// A pointer out of the table, which lies in the device's memory like all that kernels are given.
template <typename T>
using Global = T __attribute__((address_space(1)))*;
template <typename T, typename P>
__device__ __forceinline__ Global<T> global(P* p) {
  return (Global<T>)reinterpret_cast<uintptr_t>(p);
}

// 16, 8 or 4 bytes that are touched once a step, past the caches' replacement (those weights 1525 us, through the
// caches 1685; 300 tensors of 5.4 million weights in 8 bits 17.7 and 18.6).
template <typename T>
__device__ __forceinline__ T load(Global<const T> p) {
  return __builtin_nontemporal_load(p);
}
template <typename T>
__device__ __forceinline__ void store(Global<T> p, T v) {
  __builtin_nontemporal_store(v, p);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A lane's 4 gradients, n of them there.
__device__ __forceinline__ void load_grads(const ParamRecord& t, int64_t at, int n, float (&g)[4]) {
  if (t.bf16) {
    const Global<const uint16_t> q = global<const uint16_t>(t.g) + at;
    if (n == 4) {
      const u32x2 w = load<u32x2>((Global<const u32x2>)q);
      g[0] = mfma::lo_bf16(w.x), g[1] = mfma::hi_bf16(w.x), g[2] = mfma::lo_bf16(w.y), g[3] = mfma::hi_bf16(w.y);
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = j < n ? bf16_to_f32(q[j]) : 0.f;
  } else {
    const Global<const float> q = global<const float>(t.g) + at;
    if (n == 4) {
      const u32x4 w = load<u32x4>((Global<const u32x4>)q);
#pragma unroll
      for (int j = 0; j < 4; ++j) g[j] = __uint_as_float(w[j]);
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = j < n ? q[j] : 0.f;
  }
}

__device__ __forceinline__ void load_floats(const float* base, int64_t at, int n, float (&v)[4]) {
  const Global<const float> q = global<const float>(base) + at;
  if (n == 4) {
    const u32x4 w = load<u32x4>((Global<const u32x4>)q);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = j < n ? q[j] : 0.f;
}

__device__ __forceinline__ void store_floats(float* base, int64_t at, int n, const float (&v)[4]) {
  const Global<float> q = global<float>(base) + at;
  if (n == 4) {
    store<u32x4>((Global<u32x4>)q, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                                                 __float_as_uint(v[3])});
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < n) q[j] = v[j];
}

__device__ __forceinline__ void store_copy(uint16_t* base, int64_t at, int n, const float (&v)[4]) {
  const Global<uint16_t> q = global<uint16_t>(base) + at;
  if (n == 4) {
    store<u32x2>((Global<u32x2>)q, u32x2{mfma::pack2(v[0], v[1]), mfma::pack2(v[2], v[3])});
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
  const float per_unit = state8::per_unit_of<SECOND>(e);
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) w |= state8::encode<SECOND>(v[j], per_unit, random[j]) << (8 * j);
  store<uint32_t>(global<uint32_t>(static_cast<uint8_t*>(codes) + place), e == 255u ? 0u : w);
  if ((threadIdx.x & 7) == 0) global<uint8_t>(scales)[place >> 5] = (uint8_t)e;
}

// (m rate) / (sqrt(v) root + eps), to 4 roundings.  The square root's instruction takes
// normal numbers: a v below 2^-96 is scaled by 2^64, its root back.
__device__ __forceinline__ float step_of(float m, float v, const AdamArgs& a) {
  const bool tiny = v < 0x1p-96f;
  const float s = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v);
  return a.rate * m * __builtin_amdgcn_rcpf(fmaf(s, tiny ? a.root * 0x1p-32f : a.root, a.eps));
}

// A lane's part of a chunk.  WHOLE: all its elements are there.
template <bool EIGHT, bool WHOLE>
__device__ __forceinline__ void step_chunk(const AdamArgs& a, const ParamRecord& t, int64_t first, float factor) {
  constexpr int kParts = kParamChunk / kSpan;
  float p[kParts][4], g[kParts][4], m[kParts][4], v[kParts][4];
  uint32_t mc[kParts], vc[kParts], me[kParts], ve[kParts];
  int n[kParts];
  bool here[kParts];  // a lane of a group with elements; places behind a tensor's last hold zeros, and keep them
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const int64_t at = first + i * kSpan, left = t.n - at, place = t.place + at;
    n[i] = WHOLE || left >= 4 ? 4 : left > 0 ? (int)left : 0;
    here[i] = WHOLE || t.n > (EIGHT ? at & -32 : at);
    if (!here[i]) continue;
    load_grads(t, at, n[i], g[i]);
    load_floats(t.p, at, n[i], p[i]);
    if (EIGHT) {
      mc[i] = load<uint32_t>(global<const uint32_t>(static_cast<const uint8_t*>(a.m) + place));
      vc[i] = load<uint32_t>(global<const uint32_t>(static_cast<const uint8_t*>(a.v) + place));
      me[i] = a.m_scales[place >> 5], ve[i] = a.v_scales[place >> 5];
    } else {
      load_floats(static_cast<const float*>(a.m), place, 4, m[i]);
      load_floats(static_cast<const float*>(a.v), place, 4, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    if (!here[i]) continue;
    const int64_t at = first + i * kSpan, place = t.place + at;
    if (EIGHT) decode4<false>(mc[i], me[i], m[i]), decode4<true>(vc[i], ve[i], v[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // each product and sum rounded by itself, so that the states do not hang on how they were fused
#pragma clang fp contract(off)
      const float x = g[i][j] * factor;
      m[i][j] = a.beta1 * m[i][j] + a.new1 * x;
      v[i][j] = a.beta2 * v[i][j] + a.new2 * x * x;
      p[i][j] = p[i][j] - (a.decay * p[i][j] + step_of(m[i][j], v[i][j], a));
    }
    store_floats(t.p, at, n[i], p[i]);
    if (t.copy) store_copy(t.copy, at, n[i], p[i]);
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
      store_floats(static_cast<float*>(a.m), place, 4, m[i]);
      store_floats(static_cast<float*>(a.v), place, 4, v[i]);
    }
  }
}

template <bool EIGHT>
__global__ void __launch_bounds__(kThreads) step_kernel(const AdamArgs a) {
  const int64_t chunk = block_index();
  if (chunk >= a.chunks) return;
  const float factor = a.factor ? *a.factor : 1.f;
  if (factor != factor) return;  // gradients that are not finite: nothing changes
  const ParamRecord t = a.tensors[a.owner[chunk]];
  const int64_t base = (chunk - t.chunk) * kParamChunk;
  // without the checks 8 bits take 873 us instead of 922 (24 blocks of 1024 channels), 32 bits 1549 instead of 1525
  if (EIGHT && base + kParamChunk <= t.n)
    step_chunk<EIGHT, true>(a, t, base + 4 * threadIdx.x, factor);
  else
    step_chunk<EIGHT, false>(a, t, base + 4 * threadIdx.x, factor);
}

// Values of a state.  A block takes two runs of 2048 codes, of which neighbouring lanes load
// 16 of one each and swap half, so that a lane has 8 of both.
constexpr int kHalf = 8 * kThreads, kPair = 2 * kHalf;

template <bool SECOND>
__device__ __forceinline__ void decode8(uint2 c, float unit, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = state8::decode<SECOND>((j < 4 ? c.x : c.y) >> (8 * (j & 3)) & 255u, unit);
}

template <bool BF16, bool SECOND>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const uint8_t* codes, const uint8_t* scales, int64_t n, void* x) {
  constexpr int kBytes = BF16 ? 2 : 4;
  const int64_t base = block_index() * kPair, at = base + 8 * threadIdx.x;
  if (base + kPair > n) {
    for (int i = 0; i < 2; ++i)
      for (int64_t k = at + i * kHalf, j = k; j < k + 8 && j < n; ++j)
        store1<BF16>(x, j, state8::decode<SECOND>(codes[j], state8::unit_of<SECOND>(scales[j >> 5])));
    return;
  }
  const int odd = threadIdx.x & 1;
  const u32x4 w = load16(codes + at + (odd ? kHalf - 8 : 0));
  const uint8_t e[2] = {scales[at >> 5], scales[(at + kHalf) >> 5]};
  uint2 c[2] = {make_uint2(w.x, w.y), make_uint2(w.z, w.w)};
  swap_pair(odd, c[0], c[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float v[8];
    decode8<SECOND>(c[i], state8::unit_of<SECOND>(e[i]), v);
    store8_stream<BF16>(static_cast<char*>(x) + (at + i * kHalf) * kBytes, v);
  }
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

// The norm and the factor from the sum of squares.
__device__ __forceinline__ void store_norm(double squares, double most, float* norm) {
  const double x = sqrt(squares);
  norm[0] = (float)x;
  norm[1] = !(x <= 0x1.fffffffffffffp1023) ? __uint_as_float(0x7FC00000u) : x <= most ? 1.f : (float)(most / x);
}

__device__ __forceinline__ void add_square(double& x, float v) { x = fma((double)v, (double)v, x); }

// Squares of float32 values in float64: neither range nor digits are lost, whatever the count.
// A block takes kRun neighbouring chunks at a time: where they are of one tensor, all of a
// lane's loads, 16 bytes each, are in flight together (the bf16 gradients of 24 blocks of
// 1024 channels: 101 us, with 8 chunks 105, with one 157).
constexpr int kRun = 4;
template <bool BF16>
__device__ __forceinline__ void square_run(const ParamRecord& t, int64_t base, double& x, double& y) {
  constexpr int kLoads = kRun * kParamChunk / kSpan / (BF16 ? 2 : 1);
  const Global<const u32x4> q = global<const u32x4>(static_cast<const char*>(t.g) + base * (BF16 ? 2 : 4)) + threadIdx.x;
  u32x4 w[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) w[i] = load<u32x4>(q + i * kThreads);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (BF16)
        add_square(x, mfma::lo_bf16(w[i][j])), add_square(y, mfma::hi_bf16(w[i][j]));
      else
        add_square(j & 1 ? y : x, __uint_as_float(w[i][j]));
    }
  }
}

__global__ void __launch_bounds__(kThreads) squares_kernel(const ParamRecord* tensors, const int32_t* owner,
                                                           int64_t chunks, double* partial, double most, float* norm) {
  static_assert(kRun * 64 == kThreads, "a wave for each chunk of a run");
  constexpr int kAll = kRun * kParamChunk;
  double x = 0., y = 0.;
  for (int64_t run = (int64_t)blockIdx.x * kRun; run < chunks; run += (int64_t)gridDim.x * kRun) {
    const int64_t last = run + kRun <= chunks ? run + kRun - 1 : chunks - 1;
    const ParamRecord t = tensors[owner[run]];
    const int64_t base = (run - t.chunk) * kParamChunk;
    if (last == run + kRun - 1 && owner[last] == owner[run] && base + kAll <= t.n) {
      t.bf16 ? square_run<true>(t, base, x, y) : square_run<false>(t, base, x, y);
      continue;
    }
    // a wave each, with all loads in flight
    const int64_t chunk = run + (threadIdx.x >> 6);
    if (chunk > last) continue;
    const ParamRecord u = tensors[owner[chunk]];
    const int64_t first = (chunk - u.chunk) * kParamChunk + 4 * (threadIdx.x & 63);
    float g[kParamChunk / 256][4];
#pragma unroll
    for (int i = 0; i < kParamChunk / 256; ++i) {
      const int64_t at = first + i * 256, left = u.n - at;
      load_grads(u, at, left >= 4 ? 4 : left > 0 ? (int)left : 0, g[i]);
    }
#pragma unroll
    for (int i = 0; i < kParamChunk / 256; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) add_square(j & 1 ? y : x, g[i][j]);
    }
  }
  x = block_sum(x + y);
  if (threadIdx.x) return;
  if (gridDim.x == 1)
    store_norm(x, most, norm);
  else
    partial[blockIdx.x] = x;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* partial, int blocks, double most, float* norm) {
  double x = 0.;
  for (int i = threadIdx.x; i < blocks; i += kThreads) x += partial[i];
  x = block_sum(x);
  if (threadIdx.x == 0) store_norm(x, most, norm);
}

// Those gradients with 512, 1024, 2048, 4096 blocks, at two places in memory: 156 and 169 us, 99 and 120, 102 and 114,
// 104 and 113.
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
  const dim3 grid = ckpt8::grid_of((n + adamw::kPair - 1) / adamw::kPair), block(adamw::kThreads);
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

int64_t grad_norm_blocks(int64_t chunks) {
  const int64_t runs = (chunks + adamw::kRun - 1) / adamw::kRun;
  return runs <= 4 ? chunks > 0 : runs < adamw::kNormBlocks ? runs : adamw::kNormBlocks;  // one block: one launch
}

void launch_grad_norm(const ParamRecord* tensors, const int32_t* owner, int64_t chunks, double most, float* norm,
                      double* partial, hipStream_t s) {
  const int blocks = (int)grad_norm_blocks(chunks);
  if (blocks)
    hipLaunchKernelGGL(adamw::squares_kernel, dim3(blocks), dim3(adamw::kThreads), 0, s, tensors, owner, chunks, partial,
                       most, norm);
  if (blocks == 1) return;
  hipLaunchKernelGGL(adamw::norm_kernel, dim3(1), dim3(adamw::kThreads), 0, s, partial, blocks, most, norm);
}

}  // namespace strata
