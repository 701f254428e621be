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
#include <type_traits>

#include "ckpt8.h"
#include "kernels.h"

namespace strata {
namespace qkv {

using namespace ckpt8;

// Waves of a block, and heads of one kind that a wave takes.  The training tile (8 tiles,
// 16 heads and their gate): rows 720 us with 2 and 780 with 4; with codes 950 and 900 (the
// exponents of 4 heads in one piece), from codes 600 and 560; the backward 850 with 2, 930
// with 4 (registers) and 920 with 1.
constexpr int kWaves = 4, kBwdHeads = 2;

// What the forward reads and writes beside the heads
enum Mode { kRows, kRowsToCodes, kFromCodes };
constexpr int fwd_heads(int mode) { return mode == kRows ? 2 : 4; }

// The sum over the lanes that hold one head's channels.
template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  x = add(x, dpp<kSwap1>(__float_as_uint(x)));
  x = add(x, dpp<kSwap2>(__float_as_uint(x)));
  if (LANES >= 8) x = add(x, dpp<kMirror8>(__float_as_uint(x)));
  if (LANES >= 16) x = add(x, dpp<kMirror16>(__float_as_uint(x)));
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

// Group g of the row's: the heads of q, then k, v and the gate, NH (k and v: NK) << near of them each.
template <int NH, int NK, int NEAR>
__device__ __forceinline__ Work work_of(const QkvArgs& a, uint32_t tile, int g) {
  Work w;
  w.tile = tile;
  const int gq = a.groups_q, gk = a.groups_k;
  int heads = a.heads, per = NH << NEAR;
  w.kind = kQ, w.first = 0;
  if (g >= gq) {
    g -= gq, w.kind = kK, w.first = a.heads, heads = a.kv, per = NK << NEAR;
    if (g >= gk) {
      g -= gk, w.kind = kV, w.first += a.kv;
      if (g >= gk) g -= gk, w.kind = kGate, w.first += a.kv, heads = a.heads, per = NH << NEAR;
    }
  }
  w.h0 = g * per;
  w.n = min(per, heads - w.h0);
  w.first += w.h0;
  return w;
}

// A lane's place: 8 channels from 8 * sub of token t, the r-th of tile b, at position
// pos of the phase table, and of heads `slot`, slot + 2^near, ... of the wave's.  The
// wave's first token is uniform, so the divisions are scalar.
struct Place {
  int sub, slot;
  bool valid;
  int64_t t, b, r, pos;
};

template <int D, int NEAR>
__device__ __forceinline__ Place place(const QkvArgs& a, uint32_t tile) {
  constexpr int kLanes = D / 8, kSlots = 64 / kLanes;
  const uint32_t t0 = tile * (kSlots >> NEAR), b0 = div_by(t0, a.by_tile), r0 = t0 - b0 * (uint32_t)a.per_tile;
  const uint32_t p0 = r0 - div_by(r0, a.by_hw) * (uint32_t)a.hw;
  Place p;
  const uint32_t lane = threadIdx.x & 63, slot = lane / kLanes;
  p.sub = lane & (kLanes - 1);
  p.slot = slot & ((1 << NEAR) - 1);
  uint32_t j = slot >> NEAR;
  p.valid = t0 + j < (uint32_t)a.tokens;
  if (!p.valid) j = (uint32_t)a.tokens - 1 - t0;  // reads stay inside, stores are left out
  uint32_t b = b0, r = r0 + j, q = p0 + j;
  while (r >= (uint32_t)a.per_tile) r -= (uint32_t)a.per_tile, ++b;
  while (q >= (uint32_t)a.hw) q -= (uint32_t)a.hw;
  p.t = t0 + j, p.b = b, p.r = r;
  p.pos = (int64_t)b * a.hw + q;
  return p;
}

// The lane's i-th head among the wave's, and where it has none, one that is there to be
// read: loads without branches between them stay in flight together.
template <int NEAR>
__device__ __forceinline__ int head_of(const Place& p, const Work& w, int i) {
  return min(p.slot + (i << NEAR), w.n - 1);
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

// Every load of the wave has arrived.  Loads and stores share a counter: a wait that the
// compiler placed in a branch after the first store would wait for that store too.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }  // vmcnt(0) alone

// 1 / root mean square of a head, from each lane's sum of squares
template <int D>
__device__ __forceinline__ float rms_factor(float squares, float eps) {
  return rsqrtf(head_sum<D / 8>(squares) * (1.f / D) + eps);
}

// The wave's slices as they lie in memory, all loads in flight before the first is
// used: the rows' elements, or their codes and exponents.
template <bool BF16, int D, bool CODES, int NH, int NEAR, bool STREAM>
struct Slices {
  Raw8<BF16> raw[NH];
  __device__ __forceinline__ void load(const QkvArgs& a, const Place& p, const Work& w) {
    constexpr int kBytes = BF16 ? 2 : 4;
    const char* at = static_cast<const char*>(a.rows) + (p.t * a.stride + (int64_t)w.first * D + 8 * p.sub) * kBytes;
#pragma unroll
    for (int i = 0; i < NH; ++i) raw[i].template load<STREAM>(at + head_of<NEAR>(p, w, i) * D * kBytes);
  }
  __device__ __forceinline__ void arrive(const Place&) {}  // after every load of the wave
  __device__ __forceinline__ void get(int i, float (&v)[8]) const { raw[i].get(v); }
  // the lane's sum of squares
  __device__ __forceinline__ float squares(int i) const {
    float v[8], m = 0.f;
    raw[i].get(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaf(v[j], v[j], m);
    return m;
  }
  // values times f, the rms factor or 1 in the norm
  __device__ __forceinline__ void scaled(int i, float f, float (&v)[8]) const {
    raw[i].get(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= f;
  }
};

// Codes.  Of two of its slices an even lane loads its own and the next lane's 8 codes
// of the first, an odd lane the same of the second; a swap gives each lane its 8 of
// both.  Steps are powers of two, so that each result equals the rows' bit for bit while
// squares and normalised values stay normal numbers (below, each path rounds its own way).
// A step of 2^121 makes a sum of squares infinite and the factor 0: the norm's values
// are then 0 whatever the codes, and their step is taken as 0.
template <bool BF16, int D, int NH, int NEAR, bool STREAM>
struct Slices<BF16, D, true, NH, NEAR, STREAM> {
  static_assert(NH % 2 == 0, "slices are loaded two at a time");
  uint2 code[NH];
  uint8_t e[NH];
  __device__ __forceinline__ void load(const QkvArgs& a, const Place& p, const Work& w) {
    const int64_t at = p.t * a.kept + (int64_t)w.first * D;
    const int odd = p.sub & 1;
#pragma unroll
    for (int i = 0; i < NH; ++i) e[i] = a.scales[(at + head_of<NEAR>(p, w, i) * D + 8 * p.sub) >> 5];
#pragma unroll
    for (int i = 0; i + 1 < NH; i += 2) {  // of a last one without a second both lanes load the first, 16 codes each
      const u32x4 c = load16(a.codes + at + head_of<NEAR>(p, w, i + odd) * D + 8 * (p.sub - odd));
      code[i] = make_uint2(c.x, c.y), code[i + 1] = make_uint2(c.z, c.w);
    }
  }
  __device__ __forceinline__ void arrive(const Place& p) {
#pragma unroll
    for (int i = 0; i + 1 < NH; i += 2) swap_pair(p.sub & 1, code[i], code[i + 1]);
  }
  __device__ __forceinline__ void get(int i, float (&v)[8]) const { decode8(code[i], step_of(e[i]), v); }
  __device__ __forceinline__ float squares(int i) const {
    const float step = step_of(e[i]);
    return code_squares(code[i]) * step * step;
  }
  __device__ __forceinline__ void scaled(int i, float f, float (&v)[8]) const {
    decode8_times(code[i], norm_step(i), f, v);
  }
  __device__ __forceinline__ float norm_step(int i) const { return e[i] == 254 ? 0.f : step_of(e[i]); }
};

// One gate logit per head: a short row of `heads` behind the slices, moved with the
// tile's first query heads.
template <bool BF16>
using Bits = typename std::conditional<BF16, uint16_t, uint32_t>::type;

template <typename T, bool BACK>
__device__ __forceinline__ void move_logits(const QkvArgs& a, uint32_t tile, uint32_t tokens) {
  const uint32_t t0 = tile * tokens, many = tokens < 8 ? 8 : tokens;
  if (t0 % many) return;  // at least 8 tokens at a time: 16 bytes of a plane
  for (uint32_t i = threadIdx.x & 63; i < many * a.heads; i += 64) {
    const uint32_t t = t0 + i % many, h = i / many;
    if (t >= (uint32_t)a.tokens) continue;
    const int64_t b = div_by(t, a.by_tile), r = t - b * a.per_tile;
    const int64_t row = t * a.stride + a.kept + h, plane = (b * a.heads + h) * a.per_tile + r;
    if (BACK)
      static_cast<T*>(a.drows)[row] = static_cast<const T*>(a.gate)[plane];
    else
      static_cast<T*>(a.gate)[plane] = static_cast<const T*>(a.rows)[row];
  }
}

template <bool BF16, int D, int MODE, bool STREAM>
__global__ void __launch_bounds__(kWaves * 64) fwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8, kBytes = BF16 ? 2 : 4, kHeads = fwd_heads(MODE);
  const uint32_t wave = (uint32_t)block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= a.waves) return;
  const uint32_t at_tile = div_by(wave, a.by_groups);
  const Work w = work_of<kHeads, kHeads, 0>(a, at_tile, (int)(wave - at_tile * a.groups));
  const Place p = place<D, 0>(a, w.tile);
  Slices<BF16, D, MODE == kFromCodes, kHeads, 0, STREAM> in;
  in.load(a, p, w);
  const bool turn = w.kind <= kK && a.cs, norm = w.kind <= kK && a.norm;
  const float* weight = w.kind == kQ ? a.wq : a.wk;
  float c[4], s[4], wt[8];
  if (turn) load_phases<D>(a, p, c, s);
  if (norm && weight) load_weights(weight, p.sub, wt);
  loads_done();
  in.arrive(p);
  const int64_t plane = a.per_tile * D * kBytes;
  const int share = w.kind == kK || w.kind == kV ? a.share : 1;
  char* out = static_cast<char*>(w.kind == kQ ? a.q : w.kind == kK ? a.k : w.kind == kV ? a.v : a.gate) +
              (p.b * a.heads + (int64_t)w.h0 * share) * plane + (p.r * D + 8 * p.sub) * kBytes;
  uint2 code[kHeads];
  uint32_t exps = 0;  // lane `sub` of a head's lanes: the exponents of the lane's slice number `sub`
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (i >= w.n) break;
    float v[8];
    if constexpr (MODE == kRowsToCodes) {
      in.get(i, v);
      const uint32_t e = exponent_of(group_top(in.raw[i]));
      code[i] = encode8(v, e);
      const uint32_t all = quads_or<kLanes>(e << (8 * (p.sub >> 2)));
      if (p.sub == i) exps = all;
    }
    if (norm) {
      in.scaled(i, rms_factor<D>(in.squares(i), a.eps), v);
      if (weight) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= wt[j];
      }
    } else {
      in.get(i, v);
    }
    if (turn) rotate<false>(v, c, s);
    if (p.valid) {
      char* to = out + (int64_t)i * share * plane;
      for (int h = 0; h < share; ++h) store8_stream<BF16>(to + h * plane, v);
    }
  }
  if (MODE == kRowsToCodes) {
    const int64_t at = p.t * a.kept + (int64_t)w.first * D;
    const int odd = p.sub & 1;
#pragma unroll
    for (int i = 0; i < kHeads; i += 2) {
      if (i + 1 < kHeads && i + 1 < w.n) {
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
  if (MODE != kFromCodes && a.gate_dim == 1 && w.kind == kQ && w.h0 == 0)
    move_logits<Bits<BF16>, false>(a, w.tile, 64 / kLanes);
}

// The wave's sums over its tokens and heads of 8 values a lane.  Every exchange halves the
// values that a lane still holds: lanes 32 apart, then 16, then 8.  Lane l is left with
// channel 8 sub + 4 (l >> 5 & 1) + 2 (l >> 4 & 1) + (l >> 3 & 1), for head_dim 128 with
// two, in v[0] and v[1].
template <int D>
__device__ __forceinline__ void token_sums(float (&v)[8]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[j]), __float_as_uint(v[j + 4]), false, false);
    v[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[j]), __float_as_uint(v[j + 2]), false, false);
    v[j] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (D == 128) return;
  constexpr int kTurn8 = 0x128;  // row_ror:8, lanes 8 apart in a row of 16
  const bool high = lane & 8;
  v[0] = (high ? v[1] : v[0]) + __uint_as_float(dpp<kTurn8>(__float_as_uint(high ? v[0] : v[1])));
  if (D == 32) v[0] += __shfl_xor(v[0], 4);
}

// The gradient of a wave's slices, tile after tile: without NORM rotated back and copied,
// with it through the norm, dw taking up the lane's part of the weight's gradient.
// SHARED: k and v heads of several query heads, whose gradients are added; a wave then
// takes one of them, with four of its loads in flight.
template <bool BF16, int D, bool CODES, bool SHARED, int NEAR, bool NORM>
__device__ __forceinline__ void backward(const QkvArgs& a, const Work& w, float (&dw)[8]) {
  constexpr int kLanes = D / 8, kBytes = BF16 ? 2 : 4;
  const int sub = threadIdx.x & (kLanes - 1), kind = w.kind;
  const bool turn = kind <= kK && a.cs;
  const float* weight = kind == kQ ? a.wq : a.wk;
  float wt[8];
  if (NORM && weight) load_weights(weight, sub, wt);
  const int64_t plane = a.per_tile * D * kBytes;
  const int share = kind == kK || kind == kV ? a.share : 1;
  const char* from = static_cast<const char*>(kind == kQ ? a.q : kind == kK ? a.k : kind == kV ? a.v : a.gate) +
                     (int64_t)w.h0 * share * plane;
  for (uint32_t tile = w.tile; tile < a.tiles; tile += a.stride_tiles) {
    const Place p = place<D, NEAR>(a, tile);
    const char* in = from + p.b * a.heads * plane + (p.r * D + 8 * sub) * kBytes;
    Raw8<BF16> up[kBwdHeads];
#pragma unroll
    for (int i = 0; i < kBwdHeads; ++i)
      up[i].template load<true>(in + (int64_t)head_of<NEAR>(p, w, i) * share * plane);
    Slices<BF16, D, CODES, kBwdHeads, NEAR, NEAR == 0> rows;
    if (NORM) rows.load(a, p, w);
    float c[4], s[4];
    if (turn) load_phases<D>(a, p, c, s);
    const char* others = in + (int64_t)head_of<NEAR>(p, w, 0) * share * plane;  // of a shared head
    Raw8<BF16> more[3];
    if (SHARED && share > 1) {
      more[0].template load<true>(others + plane);
      if (share > 2) {
        more[1].template load<true>(others + 2 * plane);
        more[2].template load<true>(others + min(3, share - 1) * plane);
      }
    }
    loads_done();
    if (NORM) rows.arrive(p);
    char* out = static_cast<char*>(a.drows) + (p.t * a.stride + (int64_t)(w.first + p.slot) * D + 8 * sub) * kBytes;
#pragma unroll
    for (int i = 0; i < kBwdHeads; ++i) {
      if (i << NEAR >= w.n) break;
      const bool there = p.valid && p.slot + (i << NEAR) < w.n;
      float u[8];
      up[i].get(u);
      if (SHARED && share > 1 && i == 0) {
        float x[8];
        for (int h = 1; h < share; h += 3) {
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            if (h + k >= share) break;
            more[k].get(x);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] += x[j];
          }
          if (h + 3 < share) {
#pragma unroll
            for (int k = 0; k < 3; ++k) more[k].template load<true>(others + min(h + 3 + k, share - 1) * plane);
          }
        }
      }
      if (turn) rotate<true>(u, c, s);
      if (NORM) {
        float y[8];
        const float r = rms_factor<D>(rows.squares(i), a.eps);
        rows.scaled(i, r, y);
        // with y = r x, u' = r w g: dw += g y, dx = u' - y mean(u' y), r never squared: it may reach 2^74
        if (weight) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (there) dw[j] = fmaf(u[j], y[j], dw[j]);
            u[j] *= wt[j];
          }
        }
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          u[j] *= r;
          dot = fmaf(u[j], y[j], dot);
        }
        dot = head_sum<kLanes>(dot) * (1.f / D);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = fmaf(-y[j], dot, u[j]);
      }
      if (there) store8_stream<BF16>(out + (i << NEAR) * D * kBytes, u);
    }
    if (a.gate_dim == 1 && kind == kQ && w.h0 == 0)
      move_logits<Bits<BF16>, true>(a, tile, (64 / kLanes) >> NEAR);
  }
}

// Blocks [0, norm_blocks) take the heads of q and k and write a row of partial weight
// gradients each, the others those of v and the gate.
template <bool BF16, int D, bool CODES, bool SHARED, int NEAR>
__global__ void __launch_bounds__(kWaves * 64) bwd_kernel(const QkvArgs a) {
  constexpr int kLanes = D / 8;
  const int64_t block = block_index();
  const bool head = block < a.norm_blocks;
  const uint32_t in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t wave = (uint32_t)(head ? block : block - a.norm_blocks) * kWaves + in_block;
  const uint32_t at_tile = div_by(wave, head ? a.by_groups : a.by_rest);
  const int group = (int)(wave - at_tile * (head ? a.groups : a.rest)) + (head ? 0 : (int)a.groups);
  const int sub = threadIdx.x & (kLanes - 1);
  float dw[8] = {};
  int kind = kGate;
  if (at_tile < a.stride_tiles) {
    const Work w = work_of<kBwdHeads, SHARED ? 1 : kBwdHeads, NEAR>(a, at_tile, group);
    kind = w.kind;
    if (head && a.norm)
      backward<BF16, D, CODES, SHARED, NEAR, true>(a, w, dw);
    else
      backward<BF16, D, CODES, SHARED, NEAR, false>(a, w, dw);
  }
  if (!a.partial || !head) return;
  __shared__ float sums[kWaves][D];
  __shared__ int kinds[kWaves];
  token_sums<D>(dw);
  const int lane = threadIdx.x & 63;
  if (lane == 0) kinds[in_block] = kind;
  const int at = 8 * sub + 4 * (lane >> 5 & 1) + 2 * (lane >> 4 & 1);
  if (D == 128) {
    sums[in_block][at] = dw[0];
    sums[in_block][at + 1] = dw[1];
  } else if (D == 64 || !(lane & 4)) {
    sums[in_block][at + (lane >> 3 & 1)] = dw[0];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kWaves * 64) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += kinds[w] == (i < D ? kQ : kK) ? sums[w][i & (D - 1)] : 0.f;
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

static int mode_of(const QkvArgs& a) { return a.codes ? kFromCodes : a.out_codes ? kRowsToCodes : kRows; }

// Waves, two rounds of the card's, that a backward keeps when a wave takes several tiles.
constexpr int64_t kFill = 16384;

// Most neighbouring heads of a token that a wave holds beside each other (log2).  Training tile, rows 32 bytes off the
// lines, microseconds with 0, 1, 2, 3 (head_dim 64): 16 heads 1600, 1330, 1290, 1230; 8 heads 807, 647, 660, 590;
// 6 heads 509, 429; 4 heads 328, 267, 273; 2 heads 181, 152.  16 heads of 32 channels with 2, 3, 4: 680, 650, 770.
// In float32 a head is twice the lines, and gains less (rows 32 bytes off, with 0, 1, 2, 3): 16 heads, 4 tiles 1143, 1078,
// 1101, 1085; 8 tiles of 8 heads 1400, 1358, 1304, 1256; 4 heads 706, 704, 704; 2 heads 317, 320; 16 heads of 32
// channels 1352, 1271, 1234, 1231; 8 heads of 128 channels, 4 tiles 1213, 1180, 1168.
static constexpr int most_near(int d) { return d == 128 ? 2 : 3; }

static void plan(QkvArgs& a, int d, bool bf16, bool back) {
  const int nh = back ? kBwdHeads : fwd_heads(mode_of(a)), nk = back && a.heads > a.kv ? 1 : nh;
  // The backward of rows that do not start on cache lines: as many neighbouring heads of a token beside each other in
  // a wave as leave less than a tenth of the lanes without one.
  a.near = 0;
  if (back && a.stride * (bf16 ? 2 : 4) % 128) {
    const int64_t gates = a.gate_dim > 1;
    for (a.near = most_near(d); a.near > 0; --a.near) {
      const int64_t step = 1 << a.near, up_h = (a.heads + step - 1) / step * step, up_kv = (a.kv + step - 1) / step * step;
      if (10 * (up_h * (1 + gates) + 2 * up_kv) <= 11 * (int64_t)a.slices) break;
    }
  }
  const int per = 512 / d >> a.near, ph = nh << a.near, pk = nk << a.near;
  a.groups_q = (a.heads + ph - 1) / ph, a.groups_k = (a.kv + pk - 1) / pk;
  a.tiles = (uint32_t)((a.tokens + per - 1) / per);
  a.groups = a.groups_q + a.groups_k;
  a.rest = a.groups_k + (a.gate_dim > 1 ? a.groups_q : 0);
  a.share = a.heads / a.kv;
  // a block's row of partial weight gradients, 8 d bytes, against 3 KB that each of its waves moves for a head of a
  // tile: as many tiles a wave as keep it near 2 %, where the card stays full
  int64_t steps = 1;
  if (back && a.norm) {
    const int64_t fill = (int64_t)a.tiles * a.groups / kFill;
    const int held = (a.heads + (1 << a.near) - 1) >> a.near;
    const int64_t want = d / (32 * (held < nh ? held : nh));
    steps = want < fill ? want : fill;
    if (steps < 1) steps = 1;
  }
  a.stride_tiles = (uint32_t)((a.tiles + steps - 1) / steps);
  if (!back) a.groups += a.rest;
  a.waves = a.stride_tiles * a.groups;
  a.by_groups = fast_div(a.groups);
  a.by_rest = fast_div(a.rest);
  a.by_tile = fast_div(a.per_tile);
  a.by_hw = fast_div(a.hw);
  a.norm_blocks = ((int64_t)a.waves + kWaves - 1) / kWaves;
  a.blocks = back ? a.norm_blocks + ((int64_t)a.stride_tiles * a.rest + kWaves - 1) / kWaves
                  : ((int64_t)a.waves + kWaves - 1) / kWaves;
}

// Rows past the caches' replacement: where they are so many that none of them would be
// found there again, and whole cache lines of them are read at a time (16 tiles of rows,
// 4.3 GB: 1380 us so and 1410 otherwise; 0.27 GB: 89 and 83 us; off the lines 840 and 813).
static bool streams(const QkvArgs& a, int d) {
  return d >= 64 && a.stride % 64 == 0 && a.tokens * a.stride >= (int64_t)1 << 29;
}

template <bool BF16, int D>
static void run_fwd(const QkvArgs& a, hipStream_t s) {
  const dim3 grid = grid_of(a.blocks), block(kWaves * 64);
  constexpr bool kMay = BF16 && D >= 64;
  const bool stream = kMay && streams(a, D);
  switch (mode_of(a)) {
    case kRows:
      if (stream)
        hipLaunchKernelGGL((fwd_kernel<BF16, D, kRows, kMay>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((fwd_kernel<BF16, D, kRows, false>), grid, block, 0, s, a);
      break;
    case kRowsToCodes:
      if (stream)
        hipLaunchKernelGGL((fwd_kernel<BF16, D, kRowsToCodes, kMay>), grid, block, 0, s, a);
      else
        hipLaunchKernelGGL((fwd_kernel<BF16, D, kRowsToCodes, false>), grid, block, 0, s, a);
      break;
    default: hipLaunchKernelGGL((fwd_kernel<BF16, D, kFromCodes, false>), grid, block, 0, s, a);
  }
}

template <bool BF16, int D, int NEAR>
static void run_bwd(const QkvArgs& a, hipStream_t s) {
  const dim3 grid = grid_of(a.blocks), block(kWaves * 64);
  const bool shared = a.share > 1;
  if (a.codes && shared)
    hipLaunchKernelGGL((bwd_kernel<BF16, D, true, true, NEAR>), grid, block, 0, s, a);
  else if (a.codes)
    hipLaunchKernelGGL((bwd_kernel<BF16, D, true, false, NEAR>), grid, block, 0, s, a);
  else if (shared)
    hipLaunchKernelGGL((bwd_kernel<BF16, D, false, true, NEAR>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((bwd_kernel<BF16, D, false, false, NEAR>), grid, block, 0, s, a);
}

template <bool BF16, int D>
static void run_d(const QkvArgs& a, bool back, hipStream_t s) {
  if (!back) return run_fwd<BF16, D>(a, s);
  switch (a.near) {
    case 0: return run_bwd<BF16, D, 0>(a, s);
    case 1: return run_bwd<BF16, D, 1>(a, s);
    case 2: return run_bwd<BF16, D, 2>(a, s);
    default: return run_bwd<BF16, D, most_near(D)>(a, s);
  }
}

template <bool BF16>
static void run(const QkvArgs& a, int d, bool back, hipStream_t s) {
  if (d == 32) run_d<BF16, 32>(a, back, s);
  if (d == 64) run_d<BF16, 64>(a, back, s);
  if (d == 128) run_d<BF16, 128>(a, back, s);
}

// Rows that one block of the first sum takes, of at most 2^15 blocks; a second launch adds theirs.
static int sum_rows(const QkvArgs& a) {
  const int64_t span = (a.norm_blocks + (1 << 15) - 1) >> 15;
  return (int)(span < 256 ? 256 : span);
}
static int64_t sums_of(const QkvArgs& a) { return (a.norm_blocks + sum_rows(a) - 1) / sum_rows(a); }

}  // namespace qkv

void launch_qkv_heads(QkvArgs a, int d, strata_dtype dt, hipStream_t s) {
  qkv::plan(a, d, dt == STRATA_BF16, false);
  dt == STRATA_BF16 ? qkv::run<true>(a, d, false, s) : qkv::run<false>(a, d, false, s);
}

size_t qkv_bwd_partial_bytes(QkvArgs a, int d, strata_dtype dt) {
  qkv::plan(a, d, dt == STRATA_BF16, true);
  return (size_t)(a.norm_blocks + qkv::sums_of(a)) * 2 * d * sizeof(float);
}

void launch_qkv_heads_bwd(QkvArgs a, int d, strata_dtype dt, float* dwq, float* dwk, hipStream_t s) {
  qkv::plan(a, d, dt == STRATA_BF16, true);
  dt == STRATA_BF16 ? qkv::run<true>(a, d, true, s) : qkv::run<false>(a, d, true, s);
  if (!a.partial) return;
  const float* in = a.partial;
  int64_t rows = a.norm_blocks;
  if (qkv::sums_of(a) > 2) {
    float* out = a.partial + rows * 2 * d;
    const int span = qkv::sum_rows(a);
    hipLaunchKernelGGL(qkv::weight_sum_kernel, dim3(2 * d / 32, (unsigned)qkv::sums_of(a)), dim3(qkv::kSumThreads), 0, s,
                       in, rows, span, 2 * d, out, nullptr, nullptr);
    in = out, rows = qkv::sums_of(a);
  }
  hipLaunchKernelGGL(qkv::weight_sum_kernel, dim3(2 * d / 32), dim3(qkv::kSumThreads), 0, s, in, rows, (int)rows, 2 * d,
                     nullptr, dwq, dwk);
}

}  // namespace strata
