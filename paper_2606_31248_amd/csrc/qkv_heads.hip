// Projection rows [q | k | v | gate] into the attention's head layout and the
// gradient back: RMS norm with a learned scale, StereoRoPE rotation, optionally the
// rows' 8-bit form written (or read) in the same pass.
//
// Everything streams: at 64 channels a bf16 element costs 2 bytes read, 2 written
// and about 10 operations, a fifth of what the card computes in that time, so HBM
// bounds it.  A lane holds 8 channels of one head, head_dim/8 lanes a head, a wave
// 512/head_dim consecutive tokens of kHeads neighbouring heads: it reads 16 bytes a
// lane from that many rows and writes one contiguous piece (1 KB in bf16) of each
// head's plane.  The token's phases stay in registers over the heads; sums over a
// head are DPP exchanges.  Waves are numbered heads first, tokens second, and do
// little each: what is in flight is then a narrow band of rows and of every plane.
#include "ckpt8.h"
#include "kernels.h"

namespace strata {
namespace qkv {

using namespace ckpt8;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kHeads = 4;  // heads of one kind that a wave takes

// Lanes that hold one head's channels: the sum over them, and the OR.
template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  x = add(x, dpp<kSwap1>(__float_as_uint(x)));
  x = add(x, dpp<kSwap2>(__float_as_uint(x)));
  if (LANES >= 8) x = add(x, dpp<kMirror8>(__float_as_uint(x)));
  if (LANES >= 16) x = add(x, dpp<kMirror16>(__float_as_uint(x)));
  return x;
}

template <int LANES>
__device__ __forceinline__ uint32_t quads_or(uint32_t x) {
  if (LANES >= 8) x |= dpp<kMirror8>(x);
  if (LANES >= 16) x |= dpp<kMirror16>(x);
  return x;
}

// Rotate 4 pairs by (cos, sin), or back.
template <bool BACK>
__device__ __forceinline__ void rotate(float (&v)[8], const float (&c)[4], const float (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = v[2 * i], b = v[2 * i + 1], sn = BACK ? -s[i] : s[i];
    v[2 * i] = fmaf(a, c[i], -b * sn);
    v[2 * i + 1] = fmaf(a, sn, b * c[i]);
  }
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& d) {
  return d.mul ? __umulhi(n, d.mul) >> d.shift : n;
}

// A wave's work: `n` heads from h0 of one kind, whose slices of the row start at
// slice `first`, for the tokens of one tile.
enum Kind { kQ, kK, kV, kGate };
struct Work {
  uint32_t tile;
  int kind, h0, n, first;
};

__device__ __forceinline__ Work work_of(const QkvArgs& a, uint32_t wave) {
  Work w;
  w.tile = div_by(wave, a.by_groups);
  int g = (int)(wave - w.tile * a.groups);
  const int gq = (a.heads + kHeads - 1) / kHeads, gk = (a.kv + kHeads - 1) / kHeads;
  int heads = a.heads;
  w.kind = kQ, w.first = 0;
  if (g >= gq) {
    g -= gq, w.kind = kK, w.first = a.heads, heads = a.kv;
    if (g >= gk) {
      g -= gk, w.kind = kV, w.first += a.kv;
      if (g >= gk) g -= gk, w.kind = kGate, w.first += a.kv, heads = a.heads;
    }
  }
  w.h0 = g * kHeads;
  w.n = min(kHeads, heads - w.h0);
  w.first += w.h0;
  return w;
}

// A lane's place: 8 channels from 8 * sub of token t, the r-th of tile b, at
// position pos of the phase table.  The wave's first token is uniform, so the
// divisions are scalar.
struct Place {
  int sub;
  bool valid;
  int64_t t, b, r, pos;
};

template <int D>
__device__ __forceinline__ Place place(const QkvArgs& a, uint32_t tile) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const uint32_t t0 = tile * kTokens, b0 = div_by(t0, a.by_tile), r0 = t0 - b0 * (uint32_t)a.per_tile;
  const uint32_t p0 = r0 - div_by(r0, a.by_hw) * (uint32_t)a.hw;
  Place p;
  const uint32_t lane = threadIdx.x & 63;
  p.sub = lane & (kLanes - 1);
  uint32_t j = lane / kLanes;
  p.valid = t0 + j < a.tokens;
  if (!p.valid) j = (uint32_t)a.tokens - 1 - t0;  // reads stay inside, stores are left out
  uint32_t b = b0, r = r0 + j, q = p0 + j;
  while (r >= (uint32_t)a.per_tile) r -= (uint32_t)a.per_tile, ++b;
  while (q >= (uint32_t)a.hw) q -= (uint32_t)a.hw;
  p.t = t0 + j, p.b = b, p.r = r;
  p.pos = (int64_t)b * a.hw + q;
  return p;
}

template <int D>
__device__ __forceinline__ void load_phases(const QkvArgs& a, const Place& p, float (&c)[4], float (&s)[4]) {
  const float4* q = reinterpret_cast<const float4*>(a.cs + p.pos * D + 8 * p.sub);
  const float4 x = q[0], y = q[1];
  c[0] = x.x, s[0] = x.y, c[1] = x.z, s[1] = x.w, c[2] = y.x, s[2] = y.y, c[3] = y.z, s[3] = y.w;
}

__device__ __forceinline__ void load_weights(const float* w, int sub, float (&v)[8]) {
  const float4* q = reinterpret_cast<const float4*>(w + 8 * sub);
  const float4 x = q[0], y = q[1];
  v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
}

// 1 / root mean square of a head
template <int D>
__device__ __forceinline__ float rms_factor(const float (&v)[8], float eps) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaf(v[i], v[i], m);
  return rsqrtf(head_sum<D / 8>(m) * (1.f / D) + eps);
}

// The raw pieces of the wave's slices, all loads in flight before the first is used:
// 16 bytes of bf16, 32 of float32, or the slices' codes and exponents.
template <bool BF16, int D, bool CODES>
struct Slices;

template <int D>
struct Slices<true, D, false> {
  u32x4 raw[kHeads];
  __device__ __forceinline__ void load(const QkvArgs& a, const Place& p, int first, int n) {
    const char* at = static_cast<const char*>(a.rows) + (p.t * a.stride + (int64_t)first * D + 8 * p.sub) * 2;
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i < n) raw[i] = load16(at + i * D * 2);
  }
  __device__ __forceinline__ void get(int i, float (&v)[8]) const { widen(raw[i], v); }
};

template <int D>
struct Slices<false, D, false> {
  u32x4 raw[kHeads][2];
  __device__ __forceinline__ void load(const QkvArgs& a, const Place& p, int first, int n) {
    const char* at = static_cast<const char*>(a.rows) + (p.t * a.stride + (int64_t)first * D + 8 * p.sub) * 4;
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i < n) raw[i][0] = load16(at + i * D * 4), raw[i][1] = load16(at + i * D * 4 + 16);
  }
  __device__ __forceinline__ void get(int i, float (&v)[8]) const { as_floats(raw[i][0], raw[i][1], v); }
};

// Of two neighbouring slices an even lane loads its own and the next lane's 8 codes
// of the first, an odd lane the same of the second; a swap gives each lane its 8 of both.
template <bool BF16, int D>
struct Slices<BF16, D, true> {
  uint2 code[kHeads];
  uint8_t e[kHeads];
  __device__ __forceinline__ void load(const QkvArgs& a, const Place& p, int first, int n) {
    const int64_t at = p.t * a.kept + (int64_t)first * D;
    const int odd = p.sub & 1;
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (i < n) e[i] = a.scales[(at + i * D + 8 * p.sub) >> 5];
#pragma unroll
    for (int i = 0; i < kHeads; i += 2) {
      if (i + 1 < n) {
        const u32x4 c = load16(a.codes + at + (i + odd) * D + 8 * (p.sub - odd));
        code[i] = make_uint2(c.x, c.y), code[i + 1] = make_uint2(c.z, c.w);
      } else if (i < n) {
        code[i] = *reinterpret_cast<const uint2*>(a.codes + at + i * D + 8 * p.sub);
      }
    }
#pragma unroll
    for (int i = 0; i < kHeads; i += 2)
      if (i + 1 < n) swap_pair(odd, code[i], code[i + 1]);
  }
  __device__ __forceinline__ void get(int i, float (&v)[8]) const { decode8(code[i], step_of(e[i]), v); }
};

template <bool BF16, int D, bool CODES>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes, kBytes = BF16 ? 2 : 4;
  const uint32_t wave =
      (uint32_t)block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= a.waves) return;
  const Work w = work_of(a, wave);
  const Place p = place<D>(a, w.tile);
  Slices<BF16, D, CODES> in;
  in.load(a, p, w.first, w.n);
  const bool turn = w.kind <= kK && a.cs, norm = w.kind <= kK && a.norm;
  const float* weight = w.kind == kQ ? a.wq : a.wk;
  float c[4], s[4], wt[8];
  if (turn) load_phases<D>(a, p, c, s);
  if (norm && weight) load_weights(weight, p.sub, wt);
  const int64_t plane = a.per_tile * D * kBytes;
  const int share = w.kind == kK || w.kind == kV ? a.share : 1;
  char* out = static_cast<char*>(w.kind == kQ ? a.q : w.kind == kK ? a.k : w.kind == kV ? a.v : a.gate) +
              (int64_t)w.h0 * share * plane + p.b * a.heads * plane + (p.r * D + 8 * p.sub) * kBytes;
  uint2 code[kHeads];
  uint32_t exps = 0;  // lane `sub` of a head's lanes: the exponents of slice `sub`
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (i >= w.n) break;
    float v[8];
    in.get(i, v);
    if (!CODES && a.out_codes) {
      const uint32_t e = exponent_of(group_top(v));
      code[i] = encode8(v, e);
      const uint32_t all = quads_or<kLanes>(e << (8 * (p.sub >> 2)));
      if (p.sub == i) exps = all;
    }
    if (norm) {
      const float r = rms_factor<D>(v, a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= r;
      if (weight) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= wt[j];
      }
    }
    if (turn) rotate<false>(v, c, s);
    if (p.valid)
      for (int h = 0; h < share; ++h) store8_stream<BF16>(out + (i * share + h) * plane, v);
  }
  if (!CODES && a.out_codes) {
    const int64_t at = p.t * a.kept + (int64_t)w.first * D;
    const int odd = p.sub & 1;
#pragma unroll
    for (int i = 0; i < kHeads; i += 2) {
      if (i + 1 < w.n) {
        swap_pair(odd, code[i], code[i + 1]);
        if (p.valid)
          store16(a.out_codes + at + (i + odd) * D + 8 * (p.sub - odd),
                  u32x4{code[i].x, code[i].y, code[i + 1].x, code[i + 1].y});
      } else if (i < w.n && p.valid) {
        *reinterpret_cast<uint2*>(a.out_codes + at + i * D + 8 * p.sub) = code[i];
      }
    }
    if (p.valid && p.sub < w.n) {
      uint8_t* to = a.out_scales + (at >> 5) + p.sub * (D / 32);
      if (D == 32) *to = (uint8_t)exps;
      if (D == 64) *reinterpret_cast<uint16_t*>(to) = (uint16_t)exps;
      if (D == 128) *reinterpret_cast<uint32_t*>(to) = exps;
    }
  }
  // one gate logit per head: a short row of `heads` behind the slices, with the wave of the first query heads
  if (a.gate_dim == 1 && !CODES && w.kind == kQ && w.h0 == 0) {
    const uint32_t t0 = w.tile * kTokens;
    for (int i = threadIdx.x & 63; i < kTokens * a.heads; i += 64) {
      const uint32_t t = t0 + i % kTokens;
      const int h = i / kTokens;
      if (t >= a.tokens) continue;
      const int64_t b = div_by(t, a.by_tile), r = t - b * a.per_tile;
      store1<BF16>(a.gate, (b * a.heads + h) * a.per_tile + r,
                   load1<BF16>(a.rows, t * a.stride + (int64_t)a.slices * D + h));
    }
  }
}

// A wave takes `steps` token tiles, one after the other, of its heads; its block
// writes one partial sum of each weight gradient.
template <bool BF16, int D, bool CODES>
__global__ void __launch_bounds__(kThreads) bwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8, kTokens = 64 / kLanes, kBytes = BF16 ? 2 : 4;
  const int64_t block = block_index();
  const uint32_t wave = (uint32_t)block * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int sub = threadIdx.x & (kLanes - 1);
  float dw[8] = {};
  int kind = kGate;
  if (wave < a.waves) {
    Work w = work_of(a, wave);
    kind = w.kind;
    const bool turn = kind <= kK && a.cs, norm = kind <= kK && a.norm;
    const float* weight = kind == kQ ? a.wq : a.wk;
    float wt[8];
    if (norm && weight) load_weights(weight, sub, wt);
    const int64_t plane = a.per_tile * D * kBytes;
    const int share = kind == kK || kind == kV ? a.share : 1;
    const char* from = static_cast<const char*>(kind == kQ ? a.q : kind == kK ? a.k : kind == kV ? a.v : a.gate) +
                       (int64_t)w.h0 * share * plane;
    const uint32_t first_tile = w.tile * a.steps, end = min(first_tile + a.steps, a.tiles);
    for (uint32_t tile = first_tile; tile < end; ++tile) {
      const Place p = place<D>(a, tile);
      const char* in = from + p.b * a.heads * plane + (p.r * D + 8 * sub) * kBytes;
      Raw8<BF16> up[kHeads];
#pragma unroll
      for (int i = 0; i < kHeads; ++i)
        if (i < w.n) up[i].load(in + i * share * plane);
      Slices<BF16, D, CODES> rows;
      if (norm) rows.load(a, p, w.first, w.n);
      float c[4], s[4];
      if (turn) load_phases<D>(a, p, c, s);
      char* out = static_cast<char*>(a.drows) + (p.t * a.stride + (int64_t)w.first * D + 8 * sub) * kBytes;
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (i >= w.n) break;
        float u[8];
        up[i].get(u);
        for (int h = 1; h < share; ++h) {
          Raw8<BF16> more;
          more.load(in + (i * share + h) * plane);
          float x[8];
          more.get(x);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] += x[j];
        }
        if (turn) rotate<true>(u, c, s);
        if (norm) {
          float x[8];
          rows.get(i, x);
          const float r = rms_factor<D>(x, a.eps);
          float dot = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] *= r;
          if (weight) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              if (p.valid) dw[j] = fmaf(u[j], x[j], dw[j]);
              u[j] *= wt[j];
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) dot = fmaf(u[j], x[j], dot);
          dot = head_sum<kLanes>(dot) * (1.f / D);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = r * fmaf(-x[j], dot, u[j]);
        }
        if (p.valid) store8_stream<BF16>(out + i * D * kBytes, u);
      }
      if (a.gate_dim == 1 && kind == kQ && w.h0 == 0) {
        const uint32_t t0 = tile * kTokens;
        for (int i = threadIdx.x & 63; i < kTokens * a.heads; i += 64) {
          const uint32_t t = t0 + i % kTokens;
          const int h = i / kTokens;
          if (t >= a.tokens) continue;
          const int64_t b = div_by(t, a.by_tile), r = t - b * a.per_tile;
          store1<BF16>(a.drows, t * a.stride + (int64_t)a.slices * D + h,
                       load1<BF16>(a.gate, (b * a.heads + h) * a.per_tile + r));
        }
      }
    }
  }
  if (!a.partial) return;
  // the block's sums: over a wave's tokens by lane exchanges, over its waves of a kind through LDS
  __shared__ float sums[kWaves][2][D];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) dw[j] += __shfl_xor(dw[j], m);
    if ((threadIdx.x & 63) < kLanes) {
      sums[threadIdx.x >> 6][0][8 * sub + j] = kind == kQ ? dw[j] : 0.f;
      sums[threadIdx.x >> 6][1][8 * sub + j] = kind == kK ? dw[j] : 0.f;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += sums[w][i / D][i % D];
    a.partial[block * 2 * D + i] = x;
  }
}

// Sums of `rows` rows of `cols` floats, in a fixed order: block (x, y) adds rows
// [y span, y span + span) of 32 columns into row y of `out`, or into dwq and dwk.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) weight_sum_kernel(const float* __restrict__ in, int64_t rows, int span,
                                                                int cols, float* __restrict__ out,
                                                                float* __restrict__ dwq, float* __restrict__ dwk) {
  __shared__ float sums[kSumThreads / 32][32];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  const int64_t first = (int64_t)blockIdx.y * span, last = first + span < rows ? first + span : rows;
  float x[4] = {};
  int64_t i = first + lane;
  for (; i + 96 < last; i += 128) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] += in[(i + 32 * k) * cols + col];
  }
  for (; i < last; i += 32) x[0] += in[i * cols + col];
  sums[lane][threadIdx.x & 31] = (x[0] + x[1]) + (x[2] + x[3]);
  __syncthreads();
  if (lane) return;
  float y = 0.f;
#pragma unroll
  for (int k = 0; k < kSumThreads / 32; ++k) y += sums[k][threadIdx.x & 31];
  if (out)
    out[(int64_t)blockIdx.y * cols + col] = y;
  else
    (col < cols / 2 ? dwq : dwk)[col < cols / 2 ? col : col - cols / 2] = y;
}

// n / d for n < 2^31 (d = 1: no multiplier): mul = ceil(2^(31 + l) / d), 2^l >= d, so that n mul / 2^(31 + l)
// is less than 1/d above n / d.
static FastDiv fast_div(int64_t d) {
  FastDiv f;
  if (d == 1) return f;
  int l = 1;
  while (((int64_t)1 << l) < d) ++l;
  f.mul = (uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d);
  f.shift = l - 1;
  return f;
}

// Token tiles that a wave of the backward takes: one, or so many that the blocks'
// partial weight gradients (2 d floats each) stay within 4 MB.
constexpr int64_t kMostPartials = 500000;

static void plan(QkvArgs& a, int d, bool back) {
  const int per = 512 / d;
  const int gq = (a.heads + kHeads - 1) / kHeads, gk = (a.kv + kHeads - 1) / kHeads;
  a.tiles = (uint32_t)((a.tokens + per - 1) / per);
  a.groups = gq + 2 * gk + (a.gate_dim > 1 ? gq : 0);
  a.share = a.heads / a.kv;
  a.steps = 1;
  if (back && a.norm) {
    const int64_t blocks = ((int64_t)a.tiles * a.groups + kWaves - 1) / kWaves;
    const int64_t most = kMostPartials / d;
    a.steps = (uint32_t)((blocks + most - 1) / most);
  }
  a.waves = (uint32_t)((int64_t)(a.tiles + a.steps - 1) / a.steps * a.groups);
  a.by_groups = fast_div(a.groups);
  a.by_tile = fast_div(a.per_tile);
  a.by_hw = fast_div(a.hw);
}

static int64_t blocks_of(const QkvArgs& a) { return ((int64_t)a.waves + kWaves - 1) / kWaves; }

template <template <bool, int, bool> class K>
static void dispatch(bool bf16, int d, const QkvArgs& a, hipStream_t s) {
  const bool codes = a.codes != nullptr;
#define STRATA_ONE(B, D, C) \
  if (bf16 == B && d == D && codes == C) return K<B, D, C>::run(a, grid_of(blocks_of(a)), s)
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

// Rows that one block of the sum takes: a second launch adds up to 64 blocks' results.
constexpr int kSumRows = 256;

// grid_of() may round the blocks up: every one of them writes its row
static int64_t partial_rows(const QkvArgs& a) {
  const dim3 g = grid_of(blocks_of(a));
  return (int64_t)g.x * g.y;
}

}  // namespace qkv

void launch_qkv_heads(QkvArgs a, int d, strata_dtype dt, hipStream_t s) {
  qkv::plan(a, d, false);
  qkv::dispatch<qkv::Fwd>(dt == STRATA_BF16, d, a, s);
}

size_t qkv_bwd_partial_bytes(QkvArgs a, int d) {
  qkv::plan(a, d, true);
  const int64_t rows = qkv::partial_rows(a), sums = (rows + qkv::kSumRows - 1) / qkv::kSumRows;
  return (size_t)(rows + sums) * 2 * d * sizeof(float);
}

void launch_qkv_heads_bwd(QkvArgs a, int d, strata_dtype dt, float* dwq, float* dwk, hipStream_t s) {
  qkv::plan(a, d, true);
  qkv::dispatch<qkv::Bwd>(dt == STRATA_BF16, d, a, s);
  if (!a.partial) return;
  const float* in = a.partial;
  int64_t rows = qkv::partial_rows(a);
  if (rows > 2 * qkv::kSumRows) {
    const int64_t sums = (rows + qkv::kSumRows - 1) / qkv::kSumRows;
    float* out = a.partial + rows * 2 * d;
    hipLaunchKernelGGL(qkv::weight_sum_kernel, dim3(2 * d / 32, (unsigned)sums), dim3(qkv::kSumThreads), 0, s, in, rows,
                       qkv::kSumRows, 2 * d, out, nullptr, nullptr);
    in = out, rows = sums;
  }
  hipLaunchKernelGGL(qkv::weight_sum_kernel, dim3(2 * d / 32), dim3(qkv::kSumThreads), 0, s, in, rows, (int)rows, 2 * d,
                     nullptr, dwq, dwk);
}

}  // namespace strata
