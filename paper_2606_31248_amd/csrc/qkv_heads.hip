// Projection rows [q | k | v | gate] into the attention's head layout and the
// gradient back: RMS norm with a learned scale, StereoRoPE rotation, optionally the
// rows' 8-bit form written (or read) in the same pass.
//
// Everything streams: at 64 channels a bf16 element costs 2 bytes read, 2 written
// and about 10 operations, a tenth of what the card computes in that time, so HBM
// bounds it.  A lane holds 8 channels of one head, head_dim/8 lanes a head, a wave
// 512/head_dim consecutive tokens: it reads 16 bytes a lane from that many rows and
// writes them as one contiguous piece (1 KB in bf16) of the head's plane.  The
// token's phases, and the lane's 8 weights, stay in registers while the wave walks
// the heads of its tokens; sums over a head are DPP exchanges.
#include "ckpt8.h"
#include "kernels.h"

namespace strata {
namespace qkv {

using namespace ckpt8;

constexpr int kThreads = 256, kWaves = 4;

// Lanes that hold one head's channels: sum over them.
template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  x = add(x, dpp<kSwap1>(__float_as_uint(x)));
  x = add(x, dpp<kSwap2>(__float_as_uint(x)));
  if (LANES >= 8) x = add(x, dpp<kMirror8>(__float_as_uint(x)));
  if (LANES >= 16) x = add(x, dpp<kMirror16>(__float_as_uint(x)));
  return x;
}

// Rotate 4 pairs by (cos, sin), or back with sign = -1.
__device__ __forceinline__ void rotate(float (&v)[8], const float (&c)[4], const float (&s)[4], float sign) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = v[2 * i], b = v[2 * i + 1], sn = sign * s[i];
    v[2 * i] = fmaf(a, c[i], -b * sn);
    v[2 * i + 1] = fmaf(a, sn, b * c[i]);
  }
}

// A lane's place: 8 channels from 8 * sub of token t, the r-th of tile b.
struct Place {
  int sub, valid;
  int64_t t, b, r;
};

template <int D>
__device__ __forceinline__ Place place(const QkvArgs& a, int64_t tile) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  Place p;
  p.sub = threadIdx.x & (kLanes - 1);
  p.t = tile * kTokens + ((threadIdx.x & 63) / kLanes);
  p.valid = p.t < a.tokens;
  if (!p.valid) p.t = a.tokens - 1;  // reads stay inside, stores are left out
  p.b = (uint32_t)p.t / (uint32_t)a.per_tile;
  p.r = p.t - p.b * a.per_tile;
  return p;
}

template <int D>
__device__ __forceinline__ void load_phases(const QkvArgs& a, const Place& p, float (&c)[4], float (&s)[4]) {
  const int64_t pos = p.b * a.hw + (uint32_t)p.r % (uint32_t)a.hw;
  const float4* q = reinterpret_cast<const float4*>(a.cs + pos * D + 8 * p.sub);
  const float4 x = q[0], y = q[1];
  c[0] = x.x, s[0] = x.y, c[1] = x.z, s[1] = x.w, c[2] = y.x, s[2] = y.y, c[3] = y.z, s[3] = y.w;
}

__device__ __forceinline__ void load_weights(const float* w, int sub, float (&v)[8]) {
  if (w) {
    const float4* q = reinterpret_cast<const float4*>(w + 8 * sub);
    const float4 x = q[0], y = q[1];
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.f;
  }
}

// The 8 channels of row slice `part` (a head of q, k, v or the gate), from the rows or their codes.
template <bool BF16, int D, bool CODES>
__device__ __forceinline__ void load_slice(const QkvArgs& a, const Place& p, int part, float (&v)[8]) {
  if (CODES) {
    const int64_t at = p.t * a.kept + part * D + 8 * p.sub;
    decode8(*reinterpret_cast<const uint2*>(a.codes + at), step_of(a.scales[at >> 5]), v);
  } else {
    load8<BF16>(a.rows, p.t * a.stride + part * D + 8 * p.sub, v);
  }
}

// blockIdx.x: 4 waves' tokens; blockIdx.y: `span` slices of the row.
template <bool BF16, int D, bool CODES>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const int64_t tile = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const Place p = place<D>(a, tile);
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f}, wq[8], wk[8];
  if (a.cs) load_phases<D>(a, p, c, s);
  load_weights(a.wq, p.sub, wq);
  load_weights(a.wk, p.sub, wk);
  const int64_t plane = a.per_tile * D, tile_out = p.b * a.heads * plane + p.r * D + 8 * p.sub;
  const int k0 = a.heads, v0 = k0 + a.kv, g0 = v0 + a.kv, share = a.heads / a.kv;
  const int first = blockIdx.y * a.span, last = min(first + a.span, a.slices);
  for (int part = first; part < last; ++part) {
    float v[8];
    load_slice<BF16, D, CODES>(a, p, part, v);
    if (!CODES && a.out_codes) {
      const uint32_t e = exponent_of(group_top(v));
      const uint2 code = encode8(v, e);
      if (p.valid) {
        const int64_t at = p.t * a.kept + part * D + 8 * p.sub;
        *reinterpret_cast<uint2*>(a.out_codes + at) = code;
        if ((p.sub & 3) == 0) a.out_scales[at >> 5] = (uint8_t)e;
      }
    }
    if (part < v0) {
      if (a.norm) {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaf(v[i], v[i], m);
        const float rs = rsqrtf(head_sum<kLanes>(m) * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= rs * (part < k0 ? wq[i] : wk[i]);
      }
      if (a.cs) rotate(v, c, s, 1.f);
    }
    if (!p.valid) {
    } else if (part < k0 || part >= g0) {
      store8<BF16>(part < k0 ? a.q : a.gate, tile_out + (part < k0 ? part : part - g0) * plane, v);
    } else {
      void* out = part < v0 ? a.k : a.v;
      const int h0 = (part < v0 ? part - k0 : part - v0) * share;
      for (int h = h0; h < h0 + share; ++h) store8<BF16>(out, tile_out + h * plane, v);
    }
  }
  // one gate logit per head: a short row of `heads` behind the slices
  if (a.gate_dim == 1 && !CODES && blockIdx.y == 0) {
    const int lane = threadIdx.x & 63;
    for (int i = lane; i < kTokens * a.heads; i += 64) {
      const int64_t t = tile * kTokens + i % kTokens;
      const int h = i / kTokens;
      if (t >= a.tokens) continue;
      const int64_t b = (uint32_t)t / (uint32_t)a.per_tile, r = t - b * a.per_tile;
      store1<BF16>(a.gate, (b * a.heads + h) * a.per_tile + r, load1<BF16>(a.rows, t * a.stride + a.slices * D + h));
    }
  }
}

// blockIdx.x walks the token tiles with stride gridDim.x (few partial weight
// gradients), blockIdx.y: `span` slices.
template <bool BF16, int D, bool CODES>
__global__ void __launch_bounds__(kThreads) bwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const int64_t tiles = (a.tokens + kTokens - 1) / kTokens;
  const int sub = threadIdx.x & (kLanes - 1);
  float wq[8], wk[8], gq[8] = {}, gk[8] = {};
  load_weights(a.wq, sub, wq);
  load_weights(a.wk, sub, wk);
  const int64_t plane = a.per_tile * D;
  const int k0 = a.heads, v0 = k0 + a.kv, g0 = v0 + a.kv, share = a.heads / a.kv;
  const int first = blockIdx.y * a.span, last = min(first + a.span, a.slices);
  for (int64_t tile = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); tile < tiles;
       tile += (int64_t)gridDim.x * kWaves) {
    const Place p = place<D>(a, tile);
    float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.cs) load_phases<D>(a, p, c, s);
    const int64_t tile_in = p.b * a.heads * plane + p.r * D + 8 * sub;
    for (int part = first; part < last; ++part) {
      float u[8];
      if (part < k0 || part >= g0) {
        load8<BF16>(part < k0 ? a.q : a.gate, tile_in + (part < k0 ? part : part - g0) * plane, u);
      } else {
        const void* in = part < v0 ? a.k : a.v;
        const int h0 = (part < v0 ? part - k0 : part - v0) * share;
        load8<BF16>(in, tile_in + h0 * plane, u);
        for (int h = h0 + 1; h < h0 + share; ++h) {
          float w[8];
          load8<BF16>(in, tile_in + h * plane, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] += w[i];
        }
      }
      if (part < v0) {
        if (a.cs) rotate(u, c, s, -1.f);
        if (a.norm) {
          float x[8];
          load_slice<BF16, D, CODES>(a, p, part, x);
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = fmaf(x[i], x[i], m);
          const float rs = rsqrtf(head_sum<kLanes>(m) * (1.f / D) + a.eps);
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] *= rs;
            if (p.valid) {
              if (part < k0)
                gq[i] = fmaf(u[i], x[i], gq[i]);
              else
                gk[i] = fmaf(u[i], x[i], gk[i]);
            }
            u[i] *= part < k0 ? wq[i] : wk[i];
            dot = fmaf(u[i], x[i], dot);
          }
          dot = head_sum<kLanes>(dot) * (1.f / D);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = rs * fmaf(-x[i], dot, u[i]);
        }
      }
      if (p.valid) store8<BF16>(a.drows, p.t * a.stride + part * D + 8 * sub, u);
    }
    if (a.gate_dim == 1 && blockIdx.y == 0) {
      const int lane = threadIdx.x & 63;
      for (int i = lane; i < kTokens * a.heads; i += 64) {
        const int64_t t = tile * kTokens + i / a.heads;
        const int h = i % a.heads;
        if (t >= a.tokens) continue;
        const int64_t b = (uint32_t)t / (uint32_t)a.per_tile, r = t - b * a.per_tile;
        store1<BF16>(a.drows, t * a.stride + a.slices * D + h,
                     load1<BF16>(a.gate, (b * a.heads + h) * a.per_tile + r));
      }
    }
  }
  if (!a.partial) return;
  // the block's sums: over the wave's tokens by lane exchanges, over the waves through LDS
  __shared__ float sums[kWaves][2][D];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      gq[i] += __shfl_xor(gq[i], m);
      gk[i] += __shfl_xor(gk[i], m);
    }
    if ((threadIdx.x & 63) < kLanes) {
      sums[threadIdx.x >> 6][0][8 * sub + i] = gq[i];
      sums[threadIdx.x >> 6][1][8 * sub + i] = gk[i];
    }
  }
  __syncthreads();
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += sums[w][i / D][i % D];
    a.partial[block * 2 * D + i] = x;
  }
}

// dw[c] = sum over the blocks' partial sums, in a fixed order.  One block per 16 columns.
__global__ void __launch_bounds__(kThreads) weight_sum_kernel(const float* __restrict__ partial, int blocks, int d,
                                                              float* __restrict__ dwq, float* __restrict__ dwk) {
  __shared__ float sums[16][16];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
  float x = 0.f;
  for (int i = lane; i < blocks; i += 16) x += partial[(int64_t)i * 2 * d + col];
  sums[lane][threadIdx.x & 15] = x;
  __syncthreads();
  if (lane) return;
  for (int i = 1; i < 16; ++i) x += sums[i][threadIdx.x & 15];
  (col < d ? dwq : dwk)[col < d ? col : col - d] = x;
}

// Waves that keep the card busy: 8 on each of the 1024 SIMDs.
constexpr int64_t kFill = 8192;

static int64_t token_tiles(const QkvArgs& a, int d) { return (a.tokens + 512 / d - 1) / (512 / d); }

// Slices per block: all of them where the tokens alone fill the card (a token's
// phases and place are then found once), fewer where they do not.
static int span_of(const QkvArgs& a, int d) {
  const int64_t tiles = token_tiles(a, d);
  const int64_t split = (kFill + tiles - 1) / tiles;
  return (int)(split >= a.slices ? 1 : (a.slices + split - 1) / split);
}

static dim3 bwd_grid(const QkvArgs& a, int d) {
  const int64_t blocks = (token_tiles(a, d) + kWaves - 1) / kWaves;
  const int ys = (a.slices + a.span - 1) / a.span;
  const int64_t most = kFill / kWaves / ys > 0 ? kFill / kWaves / ys : 1;
  return dim3((unsigned)(blocks < most ? blocks : most), (unsigned)ys);
}

template <template <bool, int, bool> class K, typename... A>
static void dispatch(bool bf16, int d, bool codes, A... args) {
#define STRATA_ONE(B, D, C) \
  if (bf16 == B && d == D && codes == C) return K<B, D, C>::run(args...)
  STRATA_ONE(true, 32, false);
  STRATA_ONE(true, 64, false);
  STRATA_ONE(true, 128, false);
  STRATA_ONE(true, 32, true);
  STRATA_ONE(true, 64, true);
  STRATA_ONE(true, 128, true);
  STRATA_ONE(false, 32, false);
  STRATA_ONE(false, 64, false);
  STRATA_ONE(false, 128, false);
  STRATA_ONE(false, 32, true);
  STRATA_ONE(false, 64, true);
  STRATA_ONE(false, 128, true);
#undef STRATA_ONE
}

template <bool BF16, int D, bool CODES>
struct Fwd {
  static void run(const QkvArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((fwd_kernel<BF16, D, CODES>), grid, dim3(kThreads), 0, s, a);
  }
};

template <bool BF16, int D, bool CODES>
struct Bwd {
  static void run(const QkvArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((bwd_kernel<BF16, D, CODES>), grid, dim3(kThreads), 0, s, a);
  }
};

}  // namespace qkv

void launch_qkv_heads(QkvArgs a, int d, strata_dtype dt, hipStream_t s) {
  a.span = qkv::span_of(a, d);
  const int64_t blocks = (qkv::token_tiles(a, d) + qkv::kWaves - 1) / qkv::kWaves;
  const dim3 grid((unsigned)blocks, (unsigned)((a.slices + a.span - 1) / a.span));
  qkv::dispatch<qkv::Fwd>(dt == STRATA_BF16, d, a.codes != nullptr, a, grid, s);
}

size_t qkv_bwd_partial_bytes(QkvArgs a, int d) {
  a.span = qkv::span_of(a, d);
  const dim3 g = qkv::bwd_grid(a, d);
  return (size_t)g.x * g.y * 2 * d * sizeof(float);
}

void launch_qkv_heads_bwd(QkvArgs a, int d, strata_dtype dt, float* dwq, float* dwk, hipStream_t s) {
  a.span = qkv::span_of(a, d);
  const dim3 grid = qkv::bwd_grid(a, d);
  qkv::dispatch<qkv::Bwd>(dt == STRATA_BF16, d, a.codes != nullptr, a, grid, s);
  if (a.partial)
    hipLaunchKernelGGL(qkv::weight_sum_kernel, dim3(2 * d / 16), dim3(256), 0, s, a.partial, (int)(grid.x * grid.y), d,
                       dwq, dwk);
}

}  // namespace strata
