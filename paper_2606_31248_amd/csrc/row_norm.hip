// The residual stream's addition with its RMS norm, and the gradients.
//
// Both directions stream: a bf16 element costs 8 bytes forward (10 to 12 backward) and
// about 10 (20) operations, so HBM bounds them.  A lane holds 8 channels of a piece of
// 8 * LANES, a team of LANES lanes PIECES of them, so that a row is read once and stays in
// registers between its statistics and its results; rows wider than one wave are shared by
// the waves of a block, which add their sums in LDS.  A team takes several rows, with the
// channels' gate, scale and shift (backward: and their gradients' sums) in registers.
#include "ckpt8.h"
#include "kernels.h"

namespace strata {
namespace row_norm {

using namespace ckpt8;

constexpr int kWaves = 4;               // of a block, where a row fits a wave
constexpr int kMaxWaves = 8;            // of a row: 8192 channels
constexpr int kSpan = 8;                // channels of a lane's piece

// 8 elements from any address of the type's alignment, whole or the first `n` of them.
template <bool BF16>
struct Piece;
template <>
struct Piece<true> {
  typedef u32x4 __attribute__((aligned(2))) any;
  u32x4 a;
  __device__ __forceinline__ void clear() { a = u32x4{}; }
  __device__ __forceinline__ void load(const void* p) { a = *static_cast<const any*>(p); }
  __device__ __forceinline__ void load_part(const void* p, int n) {
    const uint16_t* q = static_cast<const uint16_t*>(p);
    a = u32x4{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) a[j >> 1] |= (uint32_t)q[j] << (16 * (j & 1));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { widen(a, v); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = mfma::pack2(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void store(void* p) const { *static_cast<any*>(p) = a; }
  __device__ __forceinline__ void store_part(void* p, int n) const {
    uint16_t* q = static_cast<uint16_t*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) q[j] = (uint16_t)(a[j >> 1] >> (16 * (j & 1)));
  }
};
template <>
struct Piece<false> {
  typedef u32x4 __attribute__((aligned(4))) any;
  u32x4 a, b;
  __device__ __forceinline__ void clear() { a = b = u32x4{}; }
  __device__ __forceinline__ void load(const void* p) { a = static_cast<const any*>(p)[0], b = static_cast<const any*>(p)[1]; }
  __device__ __forceinline__ void load_part(const void* p, int n) {
    const uint32_t* q = static_cast<const uint32_t*>(p);
    clear();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < n) a[j] = q[j];
      if (4 + j < n) b[j] = q[4 + j];
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { as_floats(a, b, v); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
  }
  __device__ __forceinline__ void store(void* p) const { static_cast<any*>(p)[0] = a, static_cast<any*>(p)[1] = b; }
  __device__ __forceinline__ void store_part(void* p, int n) const {
    uint32_t* q = static_cast<uint32_t*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < n) q[j] = a[j];
      if (4 + j < n) q[4 + j] = b[j];
    }
  }
};

// A lane's n channels (0 to 8) of a row.
template <bool BF16>
__device__ __forceinline__ Piece<BF16> load(const void* base, int64_t at, int n) {
  Piece<BF16> p;
  const char* q = static_cast<const char*>(base) + at * (BF16 ? 2 : 4);
  if (n == 8)
    p.load(q);
  else
    p.load_part(q, n);
  return p;
}
template <bool BF16>
__device__ __forceinline__ void store(void* base, int64_t at, int n, const Piece<BF16>& p) {
  char* q = static_cast<char*>(base) + at * (BF16 ? 2 : 4);
  if (n == 8)
    p.store(q);
  else
    p.store_part(q, n);
}

__device__ __forceinline__ void load_vector(const float* base, int64_t at, int n, float fill, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = fill;
  if (!base) return;
  const Piece<false> p = load<false>(base, at, n);
  p.get(v);
}

// The sum over a team's lanes, in every one of them.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
  x = add(x, dpp<kSwap1>(__float_as_uint(x)));
  x = add(x, dpp<kSwap2>(__float_as_uint(x)));
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
  if (LANES <= 4) x += __uint_as_float(dpp<kTurn4>(__float_as_uint(x)));
  if (LANES <= 8) x += __uint_as_float(dpp<kTurn8>(__float_as_uint(x)));
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

// A lane's place in its team, and its channels: from `first` on, `step` apart.
template <int LANES, bool BLOCK>
struct Lane {
  int team, teams, first, step;
  __device__ __forceinline__ Lane() {
    team = BLOCK ? 0 : threadIdx.x / LANES;
    teams = BLOCK ? 1 : kWaves * 64 / LANES;
    first = kSpan * (BLOCK ? threadIdx.x : threadIdx.x & (LANES - 1));
    step = kSpan * (BLOCK ? blockDim.x : LANES);
  }
  __device__ __forceinline__ int channels(int i, int width) const {
    const int left = width - first - i * step;
    return left < 0 ? 0 : left > 8 ? 8 : left;
  }
};

template <bool BF16, int LANES, int PIECES, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kMaxWaves * 64 : kWaves * 64) fwd_kernel(const NormArgs a) {
  __shared__ float sums[2][kMaxWaves];
  int turn = 0;
  const Lane<LANES, BLOCK> at;
  const int width = a.width;
  int n[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) n[i] = at.channels(i, width);
  const float inv = 1.f / width;
  const int64_t first = block_index() * at.teams * a.steps + at.team;
  int64_t held = -1;
  float gate[PIECES][8], scale[PIECES][8], shift[PIECES][8];
  for (int k = 0; k < a.steps; ++k) {
    const int64_t t = first + (int64_t)k * at.teams;
    if (t >= a.rows) break;  // a whole team; with BLOCK the whole block
    const int64_t row = t * width + at.first;
    const int64_t b = div_by((uint32_t)t, a.by_group);
    if (b != held) {
      held = b;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int64_t c = b * width + at.first + i * at.step;
        load_vector(a.gate, c, n[i], 1.f, gate[i]);
        load_vector(a.scale, c, n[i], 1.f, scale[i]);
        load_vector(a.shift, c, n[i], 0.f, shift[i]);
      }
    }
    Piece<BF16> s[PIECES], x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) s[i] = load<BF16>(a.res, row + i * at.step, n[i]);
    if (a.x) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) x[i] = load<BF16>(a.x, row + i * at.step, n[i]);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        float u[8], v[8];
        s[i].get(u);
        x[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = fmaf(gate[i][j], v[j], u[j]);
        s[i].set(u);
        store<BF16>(a.sum, row + i * at.step, n[i], s[i]);
      }
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float u[8];
      s[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaf(u[j], u[j], m);
    }
    const float r = rsqrtf(row_sum<LANES, BLOCK>(m, sums, turn) * inv + a.eps);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float u[8];
      s[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = fmaf(u[j] * r, scale[i][j], shift[i][j]);
      s[i].set(u);
      if (a.y) store<BF16>(a.y, row + i * at.step, n[i], s[i]);
      if (a.codes && n[i]) {  // whole groups: the width is a multiple of 32
        s[i].get(u);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = umax(top, __float_as_uint(u[j]) & 0x7FFFFFFFu);
        top = umax(top, dpp<kSwap1>(top));
        top = umax(top, dpp<kSwap2>(top));
        const uint32_t e = exponent_of(top);
        const int64_t c = row + i * at.step;
        *reinterpret_cast<uint2*>(a.codes + c) = encode8(u, e);
        if ((threadIdx.x & 3) == 0) a.scales[c >> 5] = (uint8_t)e;
      }
    }
  }
}

// A block takes rows of one group, [chunk * span, ...) of them, its teams in turn; it writes
// its sums for the vectors' gradients as a row of `partial`, or where it is the group's only
// block as the gradients.
template <bool BF16, int LANES, int PIECES, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kMaxWaves * 64 : kWaves * 64) bwd_kernel(const NormArgs a) {
  __shared__ float sums[2][kMaxWaves];
  int turn = 0;
  const Lane<LANES, BLOCK> at;
  const int width = a.width;
  int n[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) n[i] = at.channels(i, width);
  const float inv = 1.f / width;
  const int64_t block = block_index();
  if (block >= a.groups * a.chunks) return;
  const int64_t b = block / a.chunks, chunk = block - b * a.chunks;
  const int64_t lo = chunk * a.span, hi = lo + a.span < a.group_rows ? lo + a.span : a.group_rows;
  float gate[PIECES][8], scale[PIECES][8], dgate[PIECES][8] = {}, dscale[PIECES][8] = {}, dshift[PIECES][8] = {};
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int64_t c = b * width + at.first + i * at.step;
    load_vector(a.gate, c, n[i], 1.f, gate[i]);
    load_vector(a.scale, c, n[i], 1.f, scale[i]);
  }
  for (int64_t k = lo + at.team; k < hi; k += at.teams) {
    const int64_t row = (b * a.group_rows + k) * width + at.first;
    Piece<BF16> s[PIECES], up[PIECES], ds[PIECES], x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) s[i] = load<BF16>(a.total, row + i * at.step, n[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) up[i] = load<BF16>(a.dy, row + i * at.step, n[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      ds[i].clear();
      if (a.dsum) ds[i] = load<BF16>(a.dsum, row + i * at.step, n[i]);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      x[i].clear();
      if (a.x) x[i] = load<BF16>(a.x, row + i * at.step, n[i]);
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float v[8];
      s[i].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaf(v[j], v[j], m);
    }
    const float r = rsqrtf(row_sum<LANES, BLOCK>(m, sums, turn) * inv + a.eps);
    // with y = r s, u = r scale dy: dres = u - y mean(u y) + dsum, r never squared: it may reach 2^74
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float v[8], u[8];
      s[i].get(v);
      up[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) dot = fmaf(u[j] * scale[i][j] * r, v[j] * r, dot);
    }
    dot = row_sum<LANES, BLOCK>(dot, sums, turn) * inv;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float v[8], u[8], h[8];
      s[i].get(v);
      up[i].get(u);
      ds[i].get(h);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] *= r;
        dscale[i][j] = fmaf(u[j], v[j], dscale[i][j]);
        dshift[i][j] += u[j];
        h[j] += fmaf(-v[j], dot, u[j] * scale[i][j] * r);
      }
      s[i].set(h);
      store<BF16>(a.dres, row + i * at.step, n[i], s[i]);
      if (a.dx) {
        x[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dgate[i][j] = fmaf(h[j], v[j], dgate[i][j]);
          h[j] *= gate[i][j];
        }
        s[i].set(h);
        store<BF16>(a.dx, row + i * at.step, n[i], s[i]);
      }
    }
  }
  // the vectors' gradients one after the other: over the wave's teams, then the block's waves
  __shared__ float wide[BLOCK ? 1 : kWaves][BLOCK ? 1 : LANES * 8 * PIECES];
  int64_t row = 0;  // of `partial`
#pragma unroll
  for (int which = 0; which < 3; ++which) {
    float* out = which == 0 ? a.dgate : which == 1 ? a.dscale : a.dshift;
    if (!out) continue;
    out = a.chunks == 1 ? out + b * width : a.partial + (row++ * a.groups * a.chunks + block) * width;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      float(&d)[8] = which == 0 ? dgate[i] : which == 1 ? dscale[i] : dshift[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (BLOCK) {
          if (j < n[i]) out[at.first + i * at.step + j] = d[j];
        } else {
          const float x = teams_sum<LANES>(d[j]);
          if ((threadIdx.x & 63) < LANES) wide[threadIdx.x >> 6][at.first + i * at.step + j] = x;
        }
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

// Waves that keep the card full, and blocks of the backward, which write a row of partial sums each.
constexpr int64_t kFill = 8192, kBwdBlocks = 1024;

static int lanes_of(int width) {
  int l = 4;
  while (l < 64 && l * kSpan < width) l *= 2;
  return l;
}
static bool by_block(int width) { return width > 2 * 64 * kSpan; }
static int threads_of(int width) { return by_block(width) ? 64 * ((width + 2 * 64 * kSpan - 1) / (2 * 64 * kSpan)) : kWaves * 64; }
static int teams_of(int width) { return by_block(width) ? 1 : kWaves * 64 / lanes_of(width); }

static void plan_bwd(NormArgs& a) {
  const int teams = teams_of(a.width);
  const int64_t most = (a.group_rows + teams - 1) / teams;
  // partial sums of 16 MiB, or a block's for 12 rows, a tenth of what these move in bf16
  const int64_t room = (16 << 20) / (3 * 4 * a.width), tenth = a.rows / 12;
  int64_t want = room > tenth ? room : tenth;
  want = (want < kBwdBlocks ? want : kBwdBlocks) / a.groups;
  a.chunks = want < 1 ? 1 : want < most ? want : most;
  a.span = (a.group_rows + a.chunks - 1) / a.chunks;
  a.chunks = (a.group_rows + a.span - 1) / a.span;
}

template <bool BF16, int LANES, int PIECES, bool BLOCK>
static void start(const NormArgs& a, bool back, dim3 grid, hipStream_t s) {
  const dim3 block(threads_of(a.width));
  if (back)
    hipLaunchKernelGGL((bwd_kernel<BF16, LANES, PIECES, BLOCK>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((fwd_kernel<BF16, LANES, PIECES, BLOCK>), grid, block, 0, s, a);
}

template <bool BF16>
static void run(const NormArgs& a, bool back, dim3 grid, hipStream_t s) {
  if (by_block(a.width)) return start<BF16, 64, 2, true>(a, back, grid, s);
  switch (lanes_of(a.width)) {
    case 4: return start<BF16, 4, 1, false>(a, back, grid, s);
    case 8: return start<BF16, 8, 1, false>(a, back, grid, s);
    case 16: return start<BF16, 16, 1, false>(a, back, grid, s);
    case 32: return start<BF16, 32, 1, false>(a, back, grid, s);
    default:
      if (a.width <= 64 * kSpan) return start<BF16, 64, 1, false>(a, back, grid, s);
      return start<BF16, 64, 2, false>(a, back, grid, s);
  }
}

}  // namespace row_norm

void launch_residual_norm(NormArgs a, strata_dtype dt, hipStream_t s) {
  const int64_t teams = row_norm::teams_of(a.width), waves = a.rows * row_norm::threads_of(a.width) / 64 / teams;
  a.steps = waves / row_norm::kFill < 1 ? 1 : waves / row_norm::kFill > 8 ? 8 : (int)(waves / row_norm::kFill);
  a.by_group = fast_div(a.group_rows);
  const dim3 grid = ckpt8::grid_of((a.rows + teams * a.steps - 1) / (teams * a.steps));
  dt == STRATA_BF16 ? row_norm::run<true>(a, false, grid, s) : row_norm::run<false>(a, false, grid, s);
}

size_t residual_norm_partial_bytes(NormArgs a) {
  row_norm::plan_bwd(a);
  return a.chunks == 1 ? 0 : (size_t)(3 * a.groups * a.chunks * a.width) * sizeof(float);
}

void launch_residual_norm_bwd(NormArgs a, strata_dtype dt, hipStream_t s) {
  row_norm::plan_bwd(a);
  const dim3 grid = ckpt8::grid_of(a.groups * a.chunks);
  dt == STRATA_BF16 ? row_norm::run<true>(a, true, grid, s) : row_norm::run<false>(a, true, grid, s);
  const unsigned vectors = !!a.dgate + !!a.dscale + !!a.dshift;
  if (a.chunks == 1 || !vectors) return;
  hipLaunchKernelGGL(row_norm::sum_kernel, dim3((a.width + 31) / 32, (unsigned)a.groups, vectors),
                     dim3(row_norm::kSumThreads), 0, s, a);
}

}  // namespace strata
