// The residual stream's addition with its RMS norm, and the gradients.
//
// Both directions stream: a bf16 element costs 8 bytes forward (backward 6 to 8, with a gate
// 10 to 12) and about 10 (20) operations, so HBM bounds them.  A lane holds 8 channels of a piece of
// 8 * LANES, a team of LANES lanes PIECES of them, so that a row is read once and stays in
// registers between its statistics and its results; rows wider than one wave are shared by
// the waves of a block, which add their sums in LDS.  Training tile (2^18 rows of 1024 in
// bf16): forward 340 us, 6.3 TB/s, backward 336, 6.4, of 6.5 that a copy reaches.
#include <algorithm>

#include "ckpt8.h"
#include "kernels.h"

namespace strata {
namespace row_norm {

using namespace ckpt8;

constexpr int kWaves = 4;               // of a block, where a row fits a wave
constexpr int kMaxWaves = 8;            // of a row: 8192 channels

// A lane's channels of a piece: 4 and 4, side by side in bf16 (16 bytes), in float32 4 in
// each half of the piece, so that both are 16 bytes beside the neighbours'.  In the last
// piece of a row less of them may be there.
struct Part {
  int lo, hi;  // of the first and the second 4
};

// How a row lies: kLines, whole cache lines that are streamed; kWhole, whole 16 bytes, so
// that a lane's 8 channels, of float32 each 4 of them, are there or not; kRagged, of any width.
enum Lie { kLines, kWhole, kRagged };

// Four elements, 16 bytes of float32, from any address of the type's alignment.  Of a ragged
// row the lanes at its end load what follows too, which is the next row but behind the last;
// `keep` clears that where it would count, not here, so that the load stays in flight.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 __attribute__((aligned(4))) float_quad;
typedef u32x2 __attribute__((aligned(4))) float_pair;
template <int LIE>
__device__ __forceinline__ u32x4 load_quad(const float* p, int n, bool inside) {
  u32x4 v = {};
  if (LIE == kLines) {
    if (n) v = load16(p);
  } else if (LIE == kWhole) {
    if (n) v = *reinterpret_cast<const u32x4*>(p);
  } else if (inside) {
    v = *reinterpret_cast<const float_quad*>(p);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) v[j] = __float_as_uint(p[j]);
  }
  return v;
}
template <int LIE>
__device__ __forceinline__ void store_quad(float* p, int n, u32x4 v) {
  if (n == 4) {
    if (LIE == kLines)
      store16(p, v);
    else
      *reinterpret_cast<float_quad*>(p) = v;
  } else if (LIE == kRagged) {  // 2 and 1: instructions for a lane of a wave cost as much as for all
    if (n & 2) *reinterpret_cast<float_pair*>(p) = u32x2{v[0], v[1]};
    if (n & 1) p[n & 2] = __uint_as_float(n & 2 ? v[2] : v[0]);
  }
}

// A lane's 8 elements of a piece as they lie in memory, at `at` of `size` and `gap` behind.
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
  typedef u32x4 __attribute__((aligned(2))) any;
  u32x4 a;
  __device__ __forceinline__ void clear() { a = u32x4{}; }
  template <int LIE>
  __device__ __forceinline__ void load(const void* base, int64_t at, int, Part n, int64_t size) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    const int many = n.lo + n.hi;
    clear();
    if (LIE == kLines) {
      if (many) a = load16(p);
    } else if (LIE == kWhole) {
      if (many) a = *reinterpret_cast<const u32x4*>(p);
    } else if (at + 8 <= size) {
      a = *reinterpret_cast<const any*>(p);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < many) a[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
  }
  template <int LIE>
  __device__ __forceinline__ void keep(Part n) {
    const int many = n.lo + n.hi;
    if (LIE != kRagged) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] &= many > 2 * j + 1 ? ~0u : many > 2 * j ? 0xFFFFu : 0u;
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { widen(a, v); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = mfma::pack2(v[2 * i], v[2 * i + 1]);
  }
  template <int LIE>
  __device__ __forceinline__ void store(void* base, int64_t at, int, Part n) const {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    const int many = n.lo + n.hi;
    if (many == 8) {
      if (LIE == kLines)
        store16(p, a);
      else
        *reinterpret_cast<any*>(p) = a;
    } else if (LIE == kRagged) {  // 4, 2 and 1
      typedef u32x2 __attribute__((aligned(2))) four;
      typedef uint32_t __attribute__((aligned(2))) two;
      if (many & 4) *reinterpret_cast<four*>(p) = u32x2{a[0], a[1]};
      if (many & 2) *reinterpret_cast<two*>(p + (many & 4)) = many & 4 ? a[2] : a[0];
      if (many & 1) p[many & 6] = (uint16_t)(many & 4 ? (many & 2 ? a[3] : a[2]) : many & 2 ? a[1] : a[0]);
    }
  }
};
template <>
struct Piece<false> {
  u32x4 a, b;
  __device__ __forceinline__ void clear() { a = b = u32x4{}; }
  template <int LIE>
  __device__ __forceinline__ void load(const void* base, int64_t at, int gap, Part n, int64_t size) {
    const float* p = static_cast<const float*>(base) + at;
    a = load_quad<LIE>(p, n.lo, at + 4 <= size);
    b = load_quad<LIE>(p + gap, n.hi, at + gap + 4 <= size);
  }
  template <int LIE>
  __device__ __forceinline__ void keep(Part n) {
    if (LIE != kRagged) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = n.lo > j ? a[j] : 0u, b[j] = n.hi > j ? b[j] : 0u;
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { as_floats(a, b, v); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
  }
  template <int LIE>
  __device__ __forceinline__ void store(void* base, int64_t at, int gap, Part n) const {
    float* p = static_cast<float*>(base) + at;
    store_quad<LIE>(p, n.lo, a);
    store_quad<LIE>(p + gap, n.hi, b);
  }
};

// A lane's part of a vector, float32 and read again by other rows.  KEEP: 0 behind a ragged
// row's end, where another group's vector begins, which may be NaN.
template <int LIE, bool KEEP = false>
__device__ __forceinline__ void load_vector(const float* base, int64_t at, int gap, Part n, int64_t size, float fill,
                                            float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = fill;
  if (!base) return;
  Piece<false> p;
  p.load<LIE == kLines ? kWhole : LIE>(base, at, gap, n, size);
  if (KEEP) p.keep<LIE>(n);
  p.get(v);
}

// The sum over a team's lanes, in every one of them.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  if (LANES >= 2) x = add(x, dpp<kSwap1>(__float_as_uint(x)));
  if (LANES >= 4) x = add(x, dpp<kSwap2>(__float_as_uint(x)));
  if (LANES >= 8) x = add(x, dpp<kMirror8>(__float_as_uint(x)));
  if (LANES >= 16) x = add(x, dpp<kMirror16>(__float_as_uint(x)));
  if (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// The sum over a wave's teams, of the lanes at the same place of each.
template <int LANES>
__device__ __forceinline__ float teams_sum(float x) {
  constexpr int kTurn4 = 0x124, kTurn8 = 0x128;  // row_ror: lanes 4, 8 apart in a row of 16
  if (LANES <= 1) x += __uint_as_float(dpp<kSwap1>(__float_as_uint(x)));
  if (LANES <= 2) x += __uint_as_float(dpp<kSwap2>(__float_as_uint(x)));
  if (LANES <= 8) x += __uint_as_float(dpp<kTurn8>(__float_as_uint(x)));
  if (LANES <= 4) x += __uint_as_float(dpp<kTurn4>(__float_as_uint(x)));
  if (LANES <= 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (LANES <= 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// The sum over a row: within the team, then over the block's waves where they share the row.
// `sums` alternates between two rows of LDS, so that one barrier a sum is enough: a wave that
// writes a row again has passed the barrier that every wave reaches after reading it.
template <int LANES, bool BLOCK>
__device__ __forceinline__ float row_sum(float x, float (*sums)[kMaxWaves], int& turn) {
  x = lanes_sum<LANES>(x);
  if (!BLOCK) return x;
  const int waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) sums[turn][threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.f;
  for (int w = 0; w < waves; ++w) x += sums[turn][w];
  turn ^= 1;
  return x;
}

// A lane's place in its team, and its channels: from `first` on, the second 4 of a piece
// `gap` behind, the pieces `step` apart.
template <bool BF16, int LANES, bool BLOCK>
struct Lane {
  int team, teams, first, gap, step;
  __device__ __forceinline__ Lane() {
    const int lanes = BLOCK ? blockDim.x : LANES, lane = BLOCK ? threadIdx.x : threadIdx.x & (LANES - 1);
    team = BLOCK ? 0 : threadIdx.x / LANES;
    teams = BLOCK ? 1 : kWaves * 64 / LANES;
    first = (BF16 ? 8 : 4) * lane;
    gap = BF16 ? 4 : 4 * lanes;
    step = 8 * lanes;
  }
  __device__ __forceinline__ Part part(int i, int width) const {
    auto four = [](int left) { return left < 0 ? 0 : left > 4 ? 4 : left; };
    const int left = width - first - i * step;
    return {four(left), four(left - gap)};
  }
};

// The largest |bits| of 4 values, and over 4 and 8 neighbouring lanes.
__device__ __forceinline__ uint32_t top4(float a, float b, float c, float d) {
  auto bits = [](float x) { return __float_as_uint(x) & 0x7FFFFFFFu; };
  return umax(umax(bits(a), bits(b)), umax(bits(c), bits(d)));
}
__device__ __forceinline__ uint32_t over_quad(uint32_t t) {
  t = umax(t, dpp<kSwap1>(t));
  return umax(t, dpp<kSwap2>(t));
}
__device__ __forceinline__ uint32_t over_eight(uint32_t t) {
  t = over_quad(t);
  return umax(t, dpp<kMirror8>(t));
}

// A team takes one row, so that what is in flight is a narrow band of each tensor's rows, and
// finds the vectors in the caches.  Training tile (2^18 rows of 1024, bf16): 6.3 TB/s; 6.0
// with 256 blocks that keep the vectors in registers and load a row ahead, 5.4 with 1024.
// Ragged rows of bf16 whose vectors take many instructions to load: where there are more blocks
// than fit the card a team takes several, loading a row ahead.
template <bool BF16, int LANES, int PIECES, bool BLOCK, int LIE>
__global__ void __launch_bounds__(BLOCK ? kMaxWaves * 64 : kWaves * 64) fwd_kernel(const NormArgs a) {
  __shared__ float sums[2][kMaxWaves];
  int turn = 0;
  const Lane<BF16, LANES, BLOCK> at;
  const int width = a.width;
  Part n[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) n[i] = at.part(i, width);
  constexpr bool kSeveral = BF16 && LIE == kRagged;
  const int64_t size = a.rows * width, stride = a.blocks * at.teams;
  Piece<BF16> s[PIECES], x[PIECES], next_s[PIECES], next_x[PIECES];
  auto fetch = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) next_s[i].template load<LIE>(a.res, t * width + at.first + i * at.step, at.gap, n[i], size);
    if (!a.x) return;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) next_x[i].template load<LIE>(a.x, t * width + at.first + i * at.step, at.gap, n[i], size);
  };
  int64_t t = block_index() * at.teams + at.team, held = -1;
  float gate[PIECES][8], scale[PIECES][8], shift[PIECES][8];
  if (t < a.rows) fetch(t);
  for (; t < a.rows; t += stride) {
    const int64_t row = t * width + at.first, b = div_by((uint32_t)t, a.by_group);
    if (b != held) {
      held = b;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int64_t c = b * width + at.first + i * at.step;
        load_vector<LIE>(a.gate, c, at.gap, n[i], a.groups * width, 1.f, gate[i]);
        load_vector<LIE>(a.scale, c, at.gap, n[i], a.groups * width, 1.f, scale[i]);
        load_vector<LIE>(a.shift, c, at.gap, n[i], a.groups * width, 0.f, shift[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) s[i] = next_s[i], x[i] = next_x[i];
    if (kSeveral && t + stride < a.rows) fetch(t + stride);
    if (a.x) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        float u[8], v[8];
        s[i].get(u);
        x[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = fmaf(gate[i][j], v[j], u[j]);
        s[i].set(u);
        s[i].template store<LIE>(a.sum, row + i * at.step, at.gap, n[i]);
      }
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float u[8];
      s[i].template keep<LIE>(n[i]);
      s[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaf(u[j], u[j], m);
    }
    const float r = rsqrtf(row_sum<LANES, BLOCK>(m, sums, turn) * a.inverse + a.eps);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float u[8];
      s[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = fmaf(u[j] * r, scale[i][j], shift[i][j]);
      s[i].set(u);
      if (a.y) s[i].template store<LIE>(a.y, row + i * at.step, at.gap, n[i]);
      if (LIE != kRagged && a.codes && n[i].lo) {  // whole groups: the width is a multiple of 32
        s[i].get(u);
        const int64_t c = row + i * at.step;
        const uint32_t lo = top4(u[0], u[1], u[2], u[3]), hi = top4(u[4], u[5], u[6], u[7]);
        if (BF16) {  // 4 lanes a group
          const uint32_t e = exponent_of(over_quad(umax(lo, hi)));
          *reinterpret_cast<uint2*>(a.codes + c) = encode8(u, e);
          if ((threadIdx.x & 3) == 0) a.scales[c >> 5] = (uint8_t)e;
        } else {  // 8 lanes, of each half
          const uint32_t e = exponent_of(over_eight(lo)), f = exponent_of(over_eight(hi));
          *reinterpret_cast<uint32_t*>(a.codes + c) = encode8(u, e).x;
          if ((threadIdx.x & 7) == 0) a.scales[c >> 5] = (uint8_t)e;
          if (n[i].hi) {
            *reinterpret_cast<uint32_t*>(a.codes + c + at.gap) = encode8(u, f).y;
            if ((threadIdx.x & 7) == 0) a.scales[(c + at.gap) >> 5] = (uint8_t)f;
          }
        }
      }
    }
    if (!kSeveral) return;
  }
}

// What the backward reads of a row.
template <bool BF16, int PIECES, bool ALL>
struct Row {
  Piece<BF16> s[PIECES], up[PIECES], ds[PIECES], x[ALL ? PIECES : 1];
  template <int LIE>
  __device__ __forceinline__ void load(const NormArgs& a, int64_t row, int step, int gap, const Part (&n)[PIECES], int64_t size) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) s[i].template load<LIE>(a.total, row + i * step, gap, n[i], size);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) up[i].template load<LIE>(a.dy, row + i * step, gap, n[i], size);
    if (ALL && a.x) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) x[i].template load<LIE>(a.x, row + i * step, gap, n[i], size);
    }
    if (a.dsum) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) ds[i].template load<LIE>(a.dsum, row + i * step, gap, n[i], size);
    }
  }
};

// The blocks of a group take its rows in turn, so that together they read a narrow band of
// them, each with the next row's loads in flight behind the present one's sums.  A block
// writes its sums for the vectors' gradients as a row of `partial`, or where it is the
// group's only block as the gradients.  ALL: with a gate or the shift's gradient, else with
// the scale's gradient at most, which takes fewer registers.
template <bool BF16, int LANES, int PIECES, bool BLOCK, int LIE, bool ALL>
__global__ void __launch_bounds__(BLOCK ? kMaxWaves * 64 : kWaves * 64) bwd_kernel(const NormArgs a) {
  __shared__ float sums[2][kMaxWaves];
  int turn = 0;
  const Lane<BF16, LANES, BLOCK> at;
  const int width = a.width;
  Part n[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) n[i] = at.part(i, width);
  const int64_t block = block_index(), size = a.rows * width;
  if (block >= a.groups * a.chunks) return;
  const int64_t b = block / a.chunks, chunk = block - b * a.chunks;
  constexpr int kAll = ALL ? PIECES : 1;
  float gate[kAll][8], scale[PIECES][8], dgate[kAll][8] = {}, dscale[PIECES][8] = {}, dshift[kAll][8] = {};
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int64_t c = b * width + at.first + i * at.step;
    if (ALL) load_vector<LIE>(a.gate, c, at.gap, n[i], a.groups * width, 1.f, gate[i]);
    load_vector<LIE, true>(a.scale, c, at.gap, n[i], a.groups * width, 1.f, scale[i]);
  }
  const int64_t last = (b + 1) * a.group_rows, stride = a.chunks * at.teams;
  int64_t t = b * a.group_rows + chunk * at.teams + at.team;
  Row<BF16, PIECES, ALL> next;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) next.ds[i].clear();
  if (t < last) next.template load<LIE>(a, t * width + at.first, at.step, at.gap, n, size);
  for (; t < last; t += stride) {
    // the loads before this row's stores: both count alike, and a wait for loads behind stores waits for these too
    Row<BF16, PIECES, ALL> in = next;
    if (t + stride < last) next.template load<LIE>(a, (t + stride) * width + at.first, at.step, at.gap, n, size);
    const int64_t row = t * width + at.first;
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float v[8];
      in.s[i].template keep<LIE>(n[i]);
      in.up[i].template keep<LIE>(n[i]);
      in.s[i].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaf(v[j], v[j], m);
    }
    const float r = rsqrtf(row_sum<LANES, BLOCK>(m, sums, turn) * a.inverse + a.eps);
    // with y = r s, u = scale dy, m = mean(u y): dres = r (u - y m) + dsum, r never squared: it may reach 2^74
    float dot = 0.f, y[PIECES][8], u[PIECES][8];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      in.s[i].get(y[i]);
      in.up[i].get(u[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[i][j] *= r;
        dscale[i][j] = fmaf(u[i][j], y[i][j], dscale[i][j]);
        if (ALL) dshift[i][j] += u[i][j];
        u[i][j] *= scale[i][j];
        dot = fmaf(u[i][j], y[i][j], dot);
      }
    }
    dot = row_sum<LANES, BLOCK>(dot, sums, turn) * a.inverse;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float h[8], v[8];
      in.ds[i].get(h);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = fmaf(r, fmaf(-y[i][j], dot, u[i][j]), h[j]);
      in.s[i].set(h);
      in.s[i].template store<LIE>(a.dres, row + i * at.step, at.gap, n[i]);
      if (ALL && a.x) {
        in.x[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dgate[i][j] = fmaf(h[j], v[j], dgate[i][j]);
          h[j] *= gate[i][j];
        }
        in.s[i].set(h);
        in.s[i].template store<LIE>(a.dx, row + i * at.step, at.gap, n[i]);
      }
    }
  }
  // the vectors' gradients one after the other: over the wave's teams, then the block's waves
  __shared__ float wide[BLOCK ? 1 : kWaves][BLOCK ? 1 : LANES * 8 * PIECES];
  int64_t row = 0;  // of `partial`
#pragma unroll
  for (int which = 0; which < 3; ++which) {
    float* out = which == 0 ? a.dgate : which == 1 ? a.dscale : a.dshift;
    if (!out || (which != 1 && !ALL)) continue;
    out = a.chunks == 1 ? out + b * width : a.partial + (row++ * a.groups * a.chunks + block) * width;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float(&d)[8] = which == 0 ? dgate[ALL ? i : 0] : which == 1 ? dscale[i] : dshift[ALL ? i : 0];
      if (BLOCK) {
        Piece<false> p;
        p.set(d);
        p.template store<LIE == kLines ? kWhole : LIE>(out, at.first + i * at.step, at.gap, n[i]);
        continue;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = teams_sum<LANES>(d[j]);
        if ((threadIdx.x & 63) < LANES)
          wide[threadIdx.x >> 6][at.first + i * at.step + (j < 4 ? j : at.gap + j - 4)] = x;
      }
    }
    if (BLOCK) continue;
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += kWaves * 64) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) x += wide[w][c];
      out[c] = x;
    }
    __syncthreads();
  }
}

// The sum of each group's rows of `partial`, in a fixed order: block (x, y, z) adds those of 32 channels
// of group y for the z-th vector that has a gradient.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const NormArgs a) {
  __shared__ float sums[kSumThreads / 32][32];
  float* out = nullptr;
  int z = blockIdx.z;
  for (float* p : {a.dgate, a.dscale, a.dshift})
    if (p && z-- == 0) out = p;
  const int64_t col = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31), group = blockIdx.y;
  const int lane = threadIdx.x >> 5;
  const float* in = a.partial + ((int64_t)blockIdx.z * a.groups + group) * a.chunks * a.width + col;
  float x[4] = {};
  if (col < a.width) {
    int64_t i = lane;
    for (; i + 96 < a.chunks; i += 128) {
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += in[(i + 32 * k) * a.width];
    }
    for (; i < a.chunks; i += 32) x[0] += in[i * a.width];
  }
  sums[lane][threadIdx.x & 31] = (x[0] + x[1]) + (x[2] + x[3]);
  __syncthreads();
  if (lane || col >= a.width) return;
  float y = 0.f;
#pragma unroll
  for (int k = 0; k < kSumThreads / 32; ++k) y += sums[k][threadIdx.x & 31];
  out[group * a.width + col] = y;
}

// A launch: lanes and pieces of a row, or where it is wider than a wave takes the waves of
// its block.
struct Shape {
  int lanes, pieces, threads, teams;
};
static bool ragged(const NormArgs& a, bool bf16) { return a.width % (bf16 ? 8 : 4); }

constexpr int kCus = 256;
constexpr int kWave = 64 * 8;  // channels of a wave's piece

// Lanes of a row of `pieces` a lane: 8 lanes hold the float32 values of a group of codes.
static int lanes_of(int width, int pieces) {
  int lanes = width % 32 ? 1 : 8;
  while (lanes < 64 && lanes * 8 * pieces < width) lanes *= 2;
  return lanes;
}

// Ragged rows, of a wave's piece at most, of which the backward's 512 blocks take less than 32 turns with a piece a lane.
static bool few(const NormArgs& a, bool bf16) {
  return ragged(a, bf16) && a.width <= kWave && a.rows < 32ll * 2 * kCus * kWaves * 64 / lanes_of(a.width, 1);
}

static Shape shape_of(const NormArgs& a, bool bf16, bool back) {
  const int width = a.width;
  if (width > 2 * kWave) return {64, 2, 64 * ((width + 2 * kWave - 1) / (2 * kWave)), 1};
  // Two pieces a lane in the backward where rows are long enough for 8 lanes: half as many exchanges an element, and a
  // wave has twice as much in flight.  The forward has more waves in flight instead (rows of 512: 6.5 and 6.2 TB/s), and
  // so do few ragged rows, whose launch is short (us of the backward with one piece and with two, 512 blocks, bf16 but where
  // said: 2^16 rows of 203 24.2, 24.5, with a gate 33.9, 35.4, in float32 61.3, 67.8; 2^17 of 100 with a gate 32.3, 34.5; 2^15
  // of 501 38.8, 40.2; but 2^18 of 203 102, 90, 2^17 of 333 96.9, 77.3, 2^19 of 100 82.6, 83.5).
  const int pieces = width > 64 && back && !few(a, bf16) ? 2 : 1, lanes = lanes_of(width, pieces);
  return {lanes, lanes * 8 < width ? 2 : 1, kWaves * 64, kWaves * 64 / lanes};
}

// Blocks of the forward: a row for each team, but in ragged rows of bf16 that are short or have a gate or a shift (TB/s
// with 1024 blocks and with all: rows of 33 4.1, 3.4; with a gate, of 203 4.5, 4.1, of 1293 3.4, 3.0; of 203 without one
// 4.6, 4.7; in float32 of 33 4.6, 5.0, of 203 4.8, 5.6).
static int64_t fwd_blocks(const NormArgs& a, bool bf16) {
  const int teams = shape_of(a, bf16, false).teams;
  const int64_t all = (a.rows + teams - 1) / teams;
  return bf16 && ragged(a, bf16) && (a.width <= 64 || a.gate || a.shift) ? std::min<int64_t>(all, 1024) : all;
}

// Blocks of the backward, which write a row of partial sums each: few waves with much in flight each read faster than
// many.  A wave a SIMD where a wave takes rows (training tile, TB/s with 256, 512, 1024 blocks: 6.4, 5.8, 5.5; with a
// gate 5.9, 5.0, 5.4), two where waves wait for each other at barriers (rows of 2048: 3.6, 5.5, 6.1) but with a gate's
// two more streams and three sums (rows of 4096 5.9, 5.5, 5.3).  If rows are many, ragged ones two (rows of 201: 4.3,
// 5.0, 4.8) or, short ones with a piece a lane, four (2^20 rows of 33 in bf16: 108, 81, 65 us), and gated ones of float32
// four (5.2, 5.7, 6.0).  Ragged ones of a wave's piece at most two at the least (with 256 and 512 blocks 2^17 rows of 33 in
// bf16 18.6 and 15.9 us, 2^16 of 100 17.1 and 16.6, 2^17 of 61 in float32 24.0 and 24.6); wider ones not (2^12 rows of 999
// in float32 with a gate 24.0 and 29.2).
static int64_t bwd_blocks(const NormArgs& a, bool bf16, bool all) {
  const Shape at = shape_of(a, bf16, true);
  if (at.teams == 1) {
    const int waves = at.threads / 64, want = all ? 4 : 8;
    return waves >= want ? kCus : kCus * (want / waves);
  }
  const bool off = ragged(a, bf16);
  const int want = off ? (a.width > 64 ? 2 : 4) : all && !bf16 ? 4 : 1, least = off && a.width <= kWave ? 2 : 1;
  return kCus * (a.rows >= (int64_t)kCus * want * 8 * at.teams ? want : least);
}

static int64_t chunks_of(const NormArgs& a, bool bf16, bool all) {
  const int teams = shape_of(a, bf16, true).teams;
  const int64_t most = (a.group_rows + teams - 1) / teams;
  if (most <= 4) return 1;  // a second launch would take longer
  // partial sums of 16 MiB, or a block's for 12 rows: of three vectors a byte an element, of the 6 to 12 that these move
  // in bf16
  const int64_t room = std::max<int64_t>((16 << 20) / (3 * 4 * a.width), a.rows / 12);
  const int64_t fill = std::min(room, bwd_blocks(a, bf16, all));
  // as many for each group as fit, or one more where a fifth of the card would be idle
  int64_t want = fill / a.groups;
  if (5 * want * a.groups < 4 * fill) ++want;
  return std::min(std::max<int64_t>(want, 1), most);
}

// Rows past the caches' replacement: of whole lines, where a tensor is larger than would be found there again.  Rows of
// 1024 in bf16, forward, so and through the caches: 2^15 rows 44.9 and 39.5 us, 2^16 85 and 93, 2^17 173 and 190; in
// float32 2^14 rows 45 and 40, 2^16 177 and 190.
static bool streams(const NormArgs& a, bool bf16) {
  return a.width % 64 == 0 && a.rows * a.width * (bf16 ? 2 : 4) >= 1 << 27;
}

template <bool BF16, int LANES, int PIECES, bool BLOCK, int LIE>
static void start(const NormArgs& a, bool back, const Shape& at, hipStream_t s) {
  const dim3 grid = grid_of(back ? a.groups * a.chunks : a.blocks), block(at.threads);
  if (!back) {
    if constexpr (PIECES == 1 || LANES == 64)
      hipLaunchKernelGGL((fwd_kernel<BF16, LANES, PIECES, BLOCK, LIE>), grid, block, 0, s, a);
  } else if (a.gate || a.dshift) {
    hipLaunchKernelGGL((bwd_kernel<BF16, LANES, PIECES, BLOCK, LIE, true>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((bwd_kernel<BF16, LANES, PIECES, BLOCK, LIE, false>), grid, block, 0, s, a);
  }
}

template <bool BF16, int LIE>
static void run(const NormArgs& a, bool back, hipStream_t s) {
  const Shape at = shape_of(a, BF16, back);
  if (at.teams == 1) return start<BF16, 64, 2, true, LIE>(a, back, at, s);
  if (at.pieces == 1) {
    switch (at.lanes) {
      case 1: return start<BF16, 1, 1, false, LIE>(a, back, at, s);
      case 2: return start<BF16, 2, 1, false, LIE>(a, back, at, s);
      case 4: return start<BF16, 4, 1, false, LIE>(a, back, at, s);
      case 8: return start<BF16, 8, 1, false, LIE>(a, back, at, s);
      case 16: return start<BF16, 16, 1, false, LIE>(a, back, at, s);
      case 32: return start<BF16, 32, 1, false, LIE>(a, back, at, s);
      default: return start<BF16, 64, 1, false, LIE>(a, back, at, s);
    }
  }
  switch (at.lanes) {
    case 8: return start<BF16, 8, 2, false, LIE>(a, back, at, s);
    case 16: return start<BF16, 16, 2, false, LIE>(a, back, at, s);
    case 32: return start<BF16, 32, 2, false, LIE>(a, back, at, s);
    default: return start<BF16, 64, 2, false, LIE>(a, back, at, s);
  }
}

template <bool BF16>
static void run(const NormArgs& a, bool back, hipStream_t s) {
  if (ragged(a, BF16)) return run<BF16, kRagged>(a, back, s);
  streams(a, BF16) ? run<BF16, kLines>(a, back, s) : run<BF16, kWhole>(a, back, s);
}

}  // namespace row_norm

void launch_residual_norm(NormArgs a, strata_dtype dt, hipStream_t s) {
  a.by_group = fast_div(a.group_rows);
  a.blocks = row_norm::fwd_blocks(a, dt == STRATA_BF16);
  dt == STRATA_BF16 ? row_norm::run<true>(a, false, s) : row_norm::run<false>(a, false, s);
}

size_t residual_norm_partial_bytes(const NormArgs& a, strata_dtype dt) {
  const bool bf16 = dt == STRATA_BF16;
  const int64_t chunks = std::max(row_norm::chunks_of(a, bf16, false), row_norm::chunks_of(a, bf16, true));
  return chunks == 1 ? 0 : (size_t)(3 * a.groups * chunks * a.width) * sizeof(float);
}

void launch_residual_norm_bwd(NormArgs a, strata_dtype dt, hipStream_t s) {
  a.chunks = row_norm::chunks_of(a, dt == STRATA_BF16, a.gate || a.dshift);
  dt == STRATA_BF16 ? row_norm::run<true>(a, true, s) : row_norm::run<false>(a, true, s);
  const unsigned vectors = !!a.dgate + !!a.dscale + !!a.dshift;
  if (a.chunks == 1 || !vectors) return;
  hipLaunchKernelGGL(row_norm::sum_kernel, dim3((a.width + 31) / 32, (unsigned)a.groups, vectors),
                     dim3(row_norm::kSumThreads), 0, s, a);
}

}  // namespace strata
