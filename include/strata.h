/*
 * strata.h -- C ABI of the STRATA hot path on AMD Instinct MI355X (gfx950).
 *
 * What it computes (arxiv 2606.31248, "Scaling Storm-Resolving Atmospheric AI
 * Simulation to the Entire Planet"):
 *   - the tile-centred stereographic coordinates of every token (Sec. 3.3, Eq. 1);
 *   - StereoRoPE: axial 2D rotary embedding driven by those coordinates (Sec. 3.3);
 *   - 3D neighbourhood attention over the (level, y, x) token grid of each tile
 *     with NATTEN's border-clamped windows (Sec. 3.2), forward and backward;
 *   - the overlapping-tile stitch S = D^-1 P^T W and its extraction P
 *     (App. F, "Tile stitching", "Linear operator interpretation");
 *   - QK RMSNorm and the sigmoid output gate of the attention block (App. B.5);
 *   - around the blocks in training: the residual stream's addition and RMS norm,
 *     the norm of the gradients and AdamW over all weights (Sec. 4);
 *   - the wind vectors of each tile in its centre's East-North frame (Sec. 3.3,
 *     Eq. 2);
 *   - the Duo-grid halo padding across cube faces and the Kaiser-Bessel-derived
 *     blend window (App. F).
 *
 * Conventions shared by every call:
 *   - Pointers are DEVICE pointers owned by the caller unless stated otherwise.
 *     The library never allocates device memory and never frees caller memory.
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL = the default
 *     stream).  Arguments are validated synchronously before any launch; on a
 *     validation error nothing is launched.
 *   - Activations are [B, heads, Z, H, W, head_dim], contiguous, head_dim
 *     innermost: B tiles, Z vertical levels, H x W horizontal tokens.
 *   - Element types: STRATA_F32 (IEEE binary32) or STRATA_BF16 (bfloat16 bit
 *     patterns in uint16 storage).  Results are rounded to nearest-even.
 *   - Every call returns a strata_status; a non-OK status leaves a message
 *     retrievable with strata_last_error() on the calling thread.  Nothing
 *     throws across the ABI.  Device pointers must be 16-byte aligned.
 */
#ifndef STRATA_H_
#define STRATA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STRATA_OK = 0,
  STRATA_ERR_INVALID_ARG = 1, /* null pointer, bad size, misalignment, bad window */
  STRATA_ERR_UNSUPPORTED = 2, /* valid arguments this build has no kernel for */
  STRATA_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required */
  STRATA_ERR_HIP = 4          /* the HIP runtime reported an error at launch */
} strata_status;

typedef enum { STRATA_F32 = 0, STRATA_BF16 = 1 } strata_dtype;

/* Neighbourhood-attention problem.  Window (kz, ky, kx): odd, 1 <= k <= extent
 * on its axis, dilation 1.  A query at position i of an axis of extent L sees
 * the k positions [s, s + k) with s = min(max(i - (k-1)/2, 0), L - k): centred,
 * shifted inward at the borders, so every query sees exactly kz*ky*kx keys. */
typedef struct {
  int32_t B, heads, Z, H, W, head_dim;
  int32_t kz, ky, kx;
  float scale;        /* logit scale, > 0 (usually 1/sqrt(head_dim)) */
  strata_dtype dtype; /* element type of q, k, v, out, dout, dq, dk, dv */
} strata_na3d_desc;

/* ---- a1: stereographic tile coordinates (Sec. 3.3, Eq. 1) -----------------
 * For tile b on the equiangular cubed sphere (faces of face_cells^2 cells,
 * tokens of patch x patch cells), token (y, x) of the tile has face token
 * (tile_oy[b] + y, tile_ox[b] + x) on face tile_face[b] (0..5).  Its
 * (lat, lon) is projected stereographically about the tile centre (the point
 * at the mean angles of the tile's first and last token) and divided by
 * l_scale, Eq. 1's length sqrt(4 pi / N_total); l_scale == 0 selects
 * sqrt(4 pi / (6 face_cells^2)) (N_total = the native cells of the six faces),
 * any other value must be finite and > 0:
 *   coords[b, y, x, 0] = x_east / l_scale,  coords[b, y, x, 1] = y_north / l_scale.
 * Face f with a = tan(alpha) (columns), c = tan(beta) (rows) is the cube point
 *   0:(1,a,c) 1:(-a,1,c) 2:(-1,-a,c) 3:(a,-1,c) 4:(-c,a,1) 5:(c,a,-1).
 * Computed in float64, stored as float32.  tile_face/oy/ox: device int32[B];
 * coords: device float32[B, H, W, 2].  Tiles must fit on the face. */
strata_status strata_stereo_coords(const int32_t* tile_face, const int32_t* tile_oy,
                                   const int32_t* tile_ox, int32_t B, int32_t H, int32_t W,
                                   int32_t face_cells, int32_t patch, double l_scale,
                                   float* coords, void* stream);

/* ---- wind vectors into the tile-centre frame (Sec. 3.3, Eq. 2) -------------
 * Cuts tiles from one cube face's horizontal wind and expresses every wind
 * vector in the East-North frame at its tile's centre:
 *   v = U e + V n  with the unit East and North vectors (e, n) at the cell's
 *   (lat, lon);  v_perp = v - (v . r0) r0;  U_loc = v_perp . e0,
 *   V_loc = v_perp . n0  with (e0, n0, r0) at the tile centre.
 * field: [P, face_cells, face_cells, 2] of dtype, (U, V) per cell of face
 * `face` (0..5, orientation as in strata_stereo_coords) for P planes (levels);
 * cell (i, j) has angles alpha = -pi/4 + (j + 1/2) (pi/2)/face_cells (columns)
 * and beta likewise from the row i.  Tile t = a*ntx + b covers the Ht x Wt
 * cells from (a*stride_y, b*stride_x); its centre is the point at the mean
 * angles of its first and last cell on each axis (at a pole the frame is the
 * formula's at the computed longitude).  tiles: [nty*ntx, P, Ht, Wt, 2] of
 * dtype.  Geometry and the 2x2 rotation in float32 for bf16 data, in float64
 * for float32 data.  Tiles must fit on the face. */
strata_status strata_wind_tile_frame(const void* field, int32_t face, int32_t face_cells, int32_t nty,
                                     int32_t ntx, int32_t P, int32_t Ht, int32_t Wt, int32_t stride_y,
                                     int32_t stride_x, void* tiles, strata_dtype dtype, void* stream);

/* ---- a2: StereoRoPE phase table (Sec. 3.3) --------------------------------
 * cs[b, y, x, t] = (cos th, sin th) for pair t < head_dim/2, with
 *   th = coords[b,y,x,0] * base^(-t/(head_dim/4))               for t <  head_dim/4,
 *   th = coords[b,y,x,1] * base^(-(t-head_dim/4)/(head_dim/4))  for t >= head_dim/4.
 * Built in float64, stored as float32 pairs.  coords: float32[B, H, W, 2];
 * cs: float32[B, H, W, head_dim/2, 2].  head_dim % 4 == 0, base > 0. */
strata_status strata_stereorope_phases(const float* coords, int32_t B, int32_t H, int32_t W,
                                       int32_t head_dim, double base, float* cs, void* stream);

/* ---- a2: StereoRoPE application (Sec. 3.3) --------------------------------
 * Rotates every pair (x[2t], x[2t+1]) of every token by its phase:
 *   y[2t] = x[2t] cos - x[2t+1] sin,  y[2t+1] = x[2t] sin + x[2t+1] cos;
 * transpose != 0 rotates by the opposite angle (R^T, used for gradients).
 * All levels and heads of a column share the phase of (b, y, x).
 * x, y: [B, heads, Z, H, W, head_dim] of dtype; y may equal x (in place).
 * Arithmetic in float32. */
strata_status strata_stereorope_apply(const void* x, void* y, const float* cs, int32_t B,
                                      int32_t heads, int32_t Z, int32_t H, int32_t W,
                                      int32_t head_dim, strata_dtype dtype, int32_t transpose,
                                      void* stream);

/* ---- a3-a6: neighbourhood attention forward (Sec. 3.2) --------------------
 * For every query i (all heads, tiles, positions):
 *   s_ij = scale * <R_i q_i, R_j k_j>  over the kz*ky*kx keys j of i's window,
 *   lse_i = ln sum_j exp(s_ij),   out_i = sum_j exp(s_ij - lse_i) v_j,
 * where R is the StereoRoPE rotation from the phase table `cs` (float32
 * [B, H, W, head_dim/2, 2]), or the identity when cs == NULL.
 * q, k, v, out: [B, heads, Z, H, W, head_dim] of desc->dtype;
 * lse: float32 [B, heads, Z, H, W] (natural log) or NULL when not needed.
 * Supported: head_dim 32, 64 or 128 in either dtype.  Kernels: bf16 at
 * head_dim 64 runs on MFMA for the windows (3,7,7), (5,9,9), (9,9,9) and every
 * column window (kz,1,1) with Z <= 32 (level sweeps for (3,7,7) and (5,9,9), a
 * query-stationary kernel for (9,9,9)); bf16 at head_dim 128 on MFMA for (9,9,9);
 * every other case (f32, head_dim 32, other windows) in float32 throughout, on
 * the float32 matrix instructions.
 * Softmax and accumulation in float32.
 * Contraction precision: on the MFMA paths the logits q.k are float16 products
 * (wider mantissa than bf16) of float16 copies of the rotated, normalised and
 * scaled q and k, accumulated in float32; P.V is a float16 product (weights and
 * V in float16) on the level-sweep kernels (3x7x7, 5x9x9), a bf16 one on the
 * others; V of magnitude above 65504 then saturates and below 2^-14 keeps
 * float16's subnormal spacing.  Input range:
 * with M = max(1, 2 scale log2(e)), inputs with M |q| <= 32000 and
 * M |k| <= 32000 (q^, k^ after the QK norm) keep every float16 operand inside
 * its range; beyond that each path saturates its float16 copies (results stay
 * finite) and the paths may give different results. */
strata_status strata_na3d_fwd(const strata_na3d_desc* desc, const void* q, const void* k,
                              const void* v, const float* cs, void* out, float* lse,
                              void* stream);

/* ---- a7: neighbourhood attention backward ----------------------------------
 * Gradients of the forward above for upstream gradient dout, with the lse the
 * forward wrote and its output `out`:
 *   P_ij = exp(s_ij - lse_i),   D_i = <dout_i, out_i>,
 *   dv_j = sum_{i: j in N(i)} P_ij dout_i,    dS_ij = P_ij (<dout_i, v_j> - D_i),
 *   dq_i = R_i^T scale sum_j dS_ij R_j k_j,    dk_j = R_j^T scale sum_i dS_ij R_i q_i.
 * lse and out have to be those of these q, k and v: with others P is no softmax, and
 * weights above 2 leave the range of the float16 products (results may be infinite).
 * Deterministic (the one atomic operation is an integer maximum, whose result
 * does not depend on order).  workspace: device memory of at least
 * strata_na3d_bwd_workspace_size(desc) bytes (holds D, one word per (batch,
 * head) and, with a gate, dA), owned by the caller.
 * Kernels and input range as strata_na3d_fwd; on the MFMA paths the dS products
 * (dq, dk) are float16 with exact power-of-two scaling; P.dO and dO.V^T are
 * float16 products with dO scaled by a power of two per (batch, head) in the
 * balanced dK/dV kernel of the 9-wide windows (V then saturates at 65504 and
 * keeps float16's subnormal spacing below 2^-14, as in the level-sweep forward;
 * with a gate it takes only (batch, head)s inside these ranges, see
 * strata_na3d_bwd_ex); elsewhere they are bf16 products, P.dO with P in two bf16
 * terms in the one-block dK/dV kernel (3x7x7, and the 9-wide windows with a gate;
 * one term with a two-term dA) and with P rounded to bf16 once in the column and
 * head_dim-128 kernels. */
size_t strata_na3d_bwd_workspace_size(const strata_na3d_desc* desc);
strata_status strata_na3d_bwd(const strata_na3d_desc* desc, const void* q, const void* k,
                              const void* v, const float* cs, const void* out, const void* dout,
                              const float* lse, void* dq, void* dk, void* dv, void* workspace,
                              size_t workspace_bytes, void* stream);

/* ---- backward for callers that cannot allocate --------------------------------
 * For code under HIP graph capture, tight training loops and harnesses that
 * forbid hipMalloc: strata_na3d_bwd without a workspace.  Same arguments,
 * results and kernels as strata_na3d_bwd (plain attention, no options); D and
 * one word per (batch, head) live in a static device array of the library
 * (32 MiB + 256 KiB), one per device, held until the process ends.  Limits:
 * B*heads*Z*H*W <= 2^23 token-heads and B*heads <= 2^16, otherwise
 * STRATA_ERR_INVALID_ARG and nothing is launched.  Nothing is allocated; the
 * array's device address is looked up once per device on the first call.
 * Every call on a device shares that device's array: calls that overlap on one
 * device (two streams, two threads) race and must be ordered by the caller. */
strata_status strata_na3d_bwd_noalloc(const strata_na3d_desc* desc, const void* q, const void* k,
                                      const void* v, const float* cs, const void* out,
                                      const void* dout, const float* lse, void* dq, void* dk,
                                      void* dv, void* stream);

/* ---- QK normalisation and the output gate (App. B.5) -----------------------
 * Options of the attention block beyond plain neighbourhood attention; a
 * zero-initialised struct (or a NULL pointer) selects plain attention.
 *   qk_norm != 0: every query and key vector (one token of one head, its
 *     head_dim entries) is divided by its root mean square before the dot
 *     product, with no learnable scale:  x^ = x / sqrt(mean_e x_e^2 + eps).
 *     The norm precedes the StereoRoPE rotation (the two commute: a rotation
 *     keeps every pair's sum of squares).  eps: finite, >= 0 (with eps = 0 an
 *     all-zero vector gives inf/NaN).
 *   gate != NULL: the attention output of every (token, head) is multiplied by
 *     sigmoid(g) = 1 / (1 + exp(-g)) of the gate logits g (device memory of
 *     desc->dtype): gate_dim == 1 -> g is [B, heads, Z, H, W], one logit per
 *     token and head; gate_dim == head_dim -> g is [B, heads, Z, H, W,
 *     head_dim], one per channel.  The logits are inputs: whatever produces
 *     them (a projection of the block input) lies outside this library. */
typedef struct {
  int32_t qk_norm;
  float eps;
  const void* gate;
  int32_t gate_dim;
} strata_na3d_opts;

/* Forward with options: s_ij = scale <R_i q^_i, R_j k^_j> (q^ = q, k^ = k when
 * qk_norm == 0), lse_i = ln sum_j exp(s_ij) (the softmax's, before the gate),
 * out_i = sigmoid(g_i) * sum_j exp(s_ij - lse_i) v_j (no factor without a
 * gate).  Everything else as strata_na3d_fwd; opts == NULL is strata_na3d_fwd. */
strata_status strata_na3d_fwd_ex(const strata_na3d_desc* desc, const strata_na3d_opts* opts,
                                 const void* q, const void* k, const void* v, const float* cs,
                                 void* out, float* lse, void* stream);

/* Backward with options, for dout = d(loss)/d(out) of the gated output, with the
 * out and lse the forward wrote.  By the chain rule through the forward:
 *   gate: a = sigmoid(g), dA = a * dout, dgate = (1 - a) * dout * out per
 *     channel (gate_dim == head_dim) or (1 - a) * <dout_i, out_i>
 *     (gate_dim == 1);
 *   attention: the backward of strata_na3d_bwd on (q^, k^, v) with upstream
 *     gradient dA (its D_i = <dA_i, A_i> equals <dout_i, out_i>);
 *   norm: dx = r (dx^ - x^ mean_e(dx^_e x^_e)), r = (mean(x^2) + eps)^(-1/2),
 *     for x = q and x = k.
 * dgate: same shape and dtype as the gate, required when opts->gate is set
 * (NULL otherwise).  workspace: at least strata_na3d_bwd_ex_workspace_size(desc,
 * opts) bytes of device memory owned by the caller; it holds D and, with a
 * gate, dA (for bf16 with a logit per channel as two bf16 terms whose sum
 * carries it to ~2^-16; with one logit per token-head 2^e dO, which is exact,
 * and lse - ln f, where sigmoid(g) = f 2^e).  With a gate every product of dO and
 * V keeps bf16's range: with one logit per token-head at 5x9x9 and 9x9x9 a (batch,
 * head) takes the balanced dK/dV kernel only where 2^e dO spans less than 2^24 from
 * row to row and V's rows lie between 2^-10 and 2^16 (their largest magnitudes),
 * and the one-block kernel otherwise, as does a problem too small to fill the chip;
 * the balanced kernel's weights P (times 2^14, float16) keep their bits down to
 * 2^-28 and are 0 below 2^-39.
 * The norm is applied inside the attention kernels.  The library allocates
 * nothing. */
size_t strata_na3d_bwd_ex_workspace_size(const strata_na3d_desc* desc,
                                         const strata_na3d_opts* opts);
strata_status strata_na3d_bwd_ex(const strata_na3d_desc* desc, const strata_na3d_opts* opts,
                                 const void* q, const void* k, const void* v, const float* cs,
                                 const void* out, const void* dout, const float* lse, void* dq,
                                 void* dk, void* dv, void* dgate, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* ---- projection rows into the attention's head layout (Sec. 3.2, App. B.5) --
 * A block's projection writes one row per token (b, z, y, x), row_stride elements
 * from the next:
 *   q: heads * d | k: kv_heads * d | v: kv_heads * d | gate: heads * gate_dim
 * (d = head_dim, head innermost but for its d channels).  One pass normalises and
 * rotates the heads and writes the layout that strata_na3d_fwd(_ex) takes:
 *   q[b, h]  = R (w_q * rms(row's q head h)),
 *   k[b, h]  = R (w_k * rms(row's k head h / (heads / kv_heads))),
 *   v[b, h]  = row's v head h / (heads / kv_heads),    gate[b, h] = row's gate,
 *   rms(x) = x / sqrt(mean_e x_e^2 + eps)   (qk_norm != 0; otherwise rms(x) = x),
 * R the StereoRoPE rotation by the phase table `cs` (float32 [B, H, W, d/2, 2];
 * NULL: the identity).  The attention is then called with cs == NULL and without
 * its own norm.  w_q, w_k: float32 [d] on the device, the learned scale of the norm
 * shared by all heads, both or neither (NULL: 1); they need qk_norm.  Arithmetic in
 * float32, one rounding to dtype.  Range of the norm, here and in the two calls below:
 * a head of root mean square 2^64 / sqrt(d) and more has squares that overflow, and a
 * norm and a gradient of 0; with eps below 2^-126 a mean square below 2^-126 keeps
 * fewer digits (17 bits at a root of 2^-66) and one of 0 makes the head NaN. */
typedef struct {
  int32_t B, heads, kv_heads, Z, H, W, head_dim; /* kv_heads divides heads */
  int32_t gate_dim;   /* gate logits per head in the rows: 0 (none), 1 or head_dim */
  int64_t row_stride; /* elements, >= the row's width, a multiple of 8 */
  int32_t qk_norm;
  float eps;          /* finite, >= 0 */
  strata_dtype dtype; /* rows, q, k, v, gate and their gradients */
} strata_qkv_desc;

/* rows: [B, Z, H, W, row_stride]; q, k, v: [B, heads, Z, H, W, head_dim]; gate:
 * [B, heads, Z, H, W] (gate_dim 1) or the shape of q (gate_dim head_dim), NULL iff
 * gate_dim == 0.  codes, scales: both NULL, or the 8-bit form (strata_ckpt_pack's)
 * of the rows' first C = (heads + 2 kv_heads + (gate_dim > 1) heads) * head_dim
 * elements, written in the same pass: codes int8 [B, Z, H, W, C], scales uint8
 * [B, Z, H, W, C/32].  One-per-head gate logits stay out of it: `gate` itself,
 * 1/head_dim of q, is what a caller keeps.  head_dim 32, 64 or 128; fewer than 2^28
 * tokens.  Buffers must not overlap. */
strata_status strata_qkv_heads(const strata_qkv_desc* desc, const void* rows, const float* wq, const float* wk,
                               const float* cs, void* q, void* k, void* v, void* gate, int8_t* codes,
                               uint8_t* scales, void* stream);

/* The same from the 8-bit form: equal bit for bit to strata_qkv_heads on rows that
 * hold the values of the codes, as long as the norm stays among float32's normal
 * numbers: not for the sign of the 0 of a head whose squares overflow, for squares
 * below 2^-126 beside an eps as small, or for normalised elements below 2^-126.
 * row_stride is not used; gate must be NULL when
 * gate_dim == 1. */
strata_status strata_qkv_heads_ckpt(const strata_qkv_desc* desc, const int8_t* codes, const uint8_t* scales,
                                    const float* wq, const float* wk, const float* cs, void* q, void* k, void* v,
                                    void* gate, void* stream);

/* Gradient of the rows and of w_q, w_k for upstream gradients dq, dk, dv, dgate in
 * the head layout (the outputs of strata_na3d_bwd(_ex)).  With g = R^T dq or R^T of
 * the sum of dk over the heads that share a key head, x the row's head, y = rms(x):
 *   dw_e = sum over tokens and heads of g_e y_e,
 *   dx = r (u - y mean_e(u_e y_e)),  u = w * g,  r = (mean_e x_e^2 + eps)^(-1/2)
 * (dx = g without qk_norm); v takes the sum of its dv, the gate its dgate.
 * The rows' values come from `rows` (codes and scales NULL) or from the 8-bit form
 * (rows NULL): then the gradient is the one at the values the codes stand for.
 * drows: [B, Z, H, W, row_stride], elements behind the row's width left as they
 * were.  dwq, dwk: float32 [head_dim], written, NULL iff the weights are.  Sums in
 * float32 in a fixed order (deterministic); one rounding to dtype.  workspace: at
 * least strata_qkv_heads_bwd_workspace_size(desc) bytes of device memory with
 * weights, else it may be NULL; calls in flight at once need one each.  Buffers must
 * not overlap.  Rows that start on 128-byte lines (row_stride a multiple of 64 in
 * bf16) are written fastest: others take 1.2 to 1.5 times as long. */
size_t strata_qkv_heads_bwd_workspace_size(const strata_qkv_desc* desc);
strata_status strata_qkv_heads_bwd(const strata_qkv_desc* desc, const void* rows, const int8_t* codes,
                                   const uint8_t* scales, const float* wq, const float* wk, const float* cs,
                                   const void* dq, const void* dk, const void* dv, const void* dgate, void* drows,
                                   float* dwq, float* dwk, void* workspace, size_t workspace_bytes, void* stream);

/* ---- activations kept in 8 bits between forward and backward ----------------
 * n elements in groups of 32 consecutive ones (the last group may be short):
 * scales[g] = s, a biased exponent, and codes[i] with the value codes[i] * 2^(s - 133).
 * With A the group's largest magnitude, 2^(s - 133) is the smallest power of two for
 * which A rounds to at most 127 steps, and at least 2^-126 (s >= 7); codes are
 * rounded to nearest, ties to even: the error of an element is at most half a step.
 * For 7 < s < 254 that is at most A/127, and the rms error of normal data about 0.9 %
 * of its standard deviation.  At s = 7 it is 2^-127, whatever A; at s = 254, where
 * codes are clamped to +-127 (A >= 1.992 * 2^127), less than one step.  A group with an
 * infinity or a NaN has s = 255 and codes 0 and stands for 32 NaN.  Encoding is
 * exact arithmetic; decoded values are exact in bf16 (7 bits).
 * x: [n] of dtype; codes: int8 [n]; scales: uint8 [ceil(n / 32)]; 1 <= n < 2^40. */
strata_status strata_ckpt_pack(const void* x, int64_t n, int8_t* codes, uint8_t* scales, strata_dtype dtype,
                               void* stream);
strata_status strata_ckpt_unpack(const int8_t* codes, const uint8_t* scales, int64_t n, void* x, strata_dtype dtype,
                                 void* stream);

/* ---- the residual stream between blocks: addition and RMS norm --------------
 * How a block is entered (Sec. 3.2; conditioned as the decoder's blocks are): the branch
 * that the block before made is added to the stream, and the sum's norm is what the next
 * projection reads.  Rows of `width` contiguous elements, one a token; group_rows
 * consecutive rows (a tile, or all rows) share a gate, a scale and a shift, float32
 * [rows / group_rows, width] each, any of them NULL (gate and scale: 1, shift: 0):
 *   sum = res + gate x  (rounded to dtype),   r = (mean_c sum_c^2 + eps)^(-1/2),
 *   y   = r sum scale + shift  (rounded to dtype);
 * without x (NULL; gate and sum then too) the norm is that of res.  y, or its 8-bit form
 * (strata_ckpt_pack's of y, bit for bit: codes int8 [rows, width], scales uint8
 * [rows, width / 32], for a width of whole 32), or both; what is not wanted is NULL.
 * Arithmetic and sums in float32.  Range of the norm, here and in the backward: a row of
 * root mean square 2^64 / sqrt(width) and more has squares that overflow, a norm of 0 and
 * no gradient through it; with eps below 2^-126 a mean square below 2^-126 keeps fewer digits
 * and one of 0 makes the row NaN.
 * sum may be res or x itself; no other buffers may overlap. */
typedef struct {
  int64_t rows;       /* 1 to 2^31 - 1, rows * width below 2^40 */
  int64_t group_rows; /* divides rows; a block of the backward takes rows of one group, so groups of few are slow */
  int32_t width;      /* 1 to 8192; whole 16 bytes of dtype are fastest */
  float eps;          /* finite, >= 0 */
  strata_dtype dtype; /* x, res, sum, y and the gradients of the rows */
} strata_norm_desc;

strata_status strata_residual_norm(const strata_norm_desc* desc, const void* x, const float* gate, const void* res,
                                   const float* scale, const float* shift, void* sum, void* y, int8_t* codes,
                                   uint8_t* scales, void* stream);

/* The gradients, for dy = d/dy and dsum = d/dsum (what the stream's later uses gave; NULL:
 * 0).  sum: the forward's (without x: its res).  With n = r sum, u = r scale dy:
 *   dres = u - n mean_c(u_c n_c) + dsum,            dx = gate dres,
 *   dscale = sum_t dy n,   dshift = sum_t dy,       dgate = sum_t dres x,
 * sums over the rows t of a group, in float32 in a fixed order (deterministic), off by at most
 * (rows / 128 + 512) 2^-24 of the sum of their terms' magnitudes, for up to 1024 channels
 * (rows / 800 + 512) 2^-24; dres and dx rounded once, dgate of the unrounded dres.  Without a gate dx is dres (pass NULL); with
 * one x, dx and dgate are needed.  dscale: needed with scale, NULL without; dshift: NULL if
 * it is not wanted.  dgate, dscale, dshift: float32 [rows / group_rows, width], written.
 * workspace: at least strata_residual_norm_bwd_workspace_size(desc) bytes (may be 0) where
 * one of the three is wanted, else it may be NULL; calls in flight at once need one each.
 * dres may be dsum or dy itself and dx may be x; no other buffers may overlap. */
size_t strata_residual_norm_bwd_workspace_size(const strata_norm_desc* desc);
strata_status strata_residual_norm_bwd(const strata_norm_desc* desc, const void* sum, const void* x, const float* gate,
                                       const float* scale, const void* dy, const void* dsum, void* dres, void* dx,
                                       float* dgate, float* dscale, float* dshift, void* workspace,
                                       size_t workspace_bytes, void* stream);

/* ---- the update of the weights: norm of the gradients, AdamW ----------------
 * A list of tensors: n elements each (0 allowed), float32 weights p, a gradient g of
 * float32 or bf16 (NULL: none, the tensor is left as it is), and a bf16 copy of the
 * weights for the model to use (NULL: none).  Device pointers, 16-byte aligned.  The
 * states m and v of all tensors lie in one buffer each, in the list's order: tensor i
 * takes n_i places from place_i, place_(i+1) = place_i + n_i rounded up to whole 32; the
 * places between are zeros.  strata_params_table writes a table of the list into HOST
 * memory of strata_params_bytes(tensors, count) bytes and fills *params but for `table`:
 * the caller copies the bytes to the device, sets params->table to the copy and keeps it,
 * the tensors and their addresses as long as the list is used.  p and copy may overlap
 * neither each other nor a gradient. */
typedef struct {
  float* p;
  const void* g;
  uint16_t* copy;
  int64_t n;
  strata_dtype grad_dtype;
} strata_param;

typedef struct {
  const void* table; /* DEVICE */
  int64_t tensors;
  int64_t chunks;    /* pieces of work */
  int64_t places;    /* elements of each state */
} strata_params;

size_t strata_params_bytes(const strata_param* tensors, int64_t count); /* 0: a bad list */
strata_status strata_params_table(const strata_param* tensors, int64_t count, void* table, size_t table_bytes,
                                  strata_params* params);

/* norm[0] = N, the square root of the sum of the squares of all gradients, norm[1] =
 * min(1, max_norm / N): what clips them (1 for N = 0; NaN where a gradient is not finite).
 * norm: float32 [2] on the device.  Sums in float64 in a fixed order; no gradient is too
 * large or small for it (norm[0] itself rounds to float32).  max_norm > 0, infinity: no
 * clipping.  workspace: strata_grad_norm_workspace_size(params) bytes (may be 0); calls in
 * flight at once need one each. */
size_t strata_grad_norm_workspace_size(const strata_params* params);
strata_status strata_grad_norm(const strata_params* params, double max_norm, float* norm, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Step number `step` (1 is the first) of AdamW on every tensor with a gradient: g' =
 * factor g (factor: NULL or one float on the device, 4-byte aligned, e.g. norm + 1; NaN:
 * nothing is changed),
 *   m <- beta1 m + (1 - beta1) g',          v <- beta2 v + (1 - beta2) g'^2,
 *   p <- p - lr (weight_decay p + (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)),
 * copy = p rounded.  In float32; m and v with every product and sum rounded by itself.
 * States: float32 (m_scales, v_scales NULL), or 8 bits: m, v uint8 [places], scales uint8
 * [places / 32], both zeros at the start, for lists of less than 2^32 places.  With E the
 * group's scale: a code c of m has a sign (bit 7) and magnitude k = c mod 128, one of v the
 * magnitude k = c, and stands for f(k) 2^(max(E - U, 1) - 127), U = 17 (m) or 33 (v), f(k) =
 * k below 8 and (8 + k mod 8) 2^(k div 8 - 1) above: 3 bits behind the leading one down to 8
 * units.  E is the biased exponent of the group's largest value after the step (one
 * more from 1.875 times the power of two on), at least U + 1 and at most 254, where the
 * largest code stands for all above it.  A value is rounded to one of its
 * two neighbours, up with the probability of its distance to the lower, so that a state
 * moves by less than a code's step (beta2 = 0.999 moves v by a thousandth) in the mean as it
 * should; v above 0 keeps at least code 1.  The random numbers are a hash of (seed, place):
 * give every step another seed.  A group with an infinity or a NaN has scale 255 and codes
 * 0 and stands for 32 NaN.
 * lr, step and seed are of the call: a captured call repeats them. */
typedef struct {
  double lr, beta1, beta2, eps, weight_decay; /* >= 0, beta < 1, eps >= 2^-126, finite */
  int64_t step;                               /* >= 1 */
  uint64_t seed;                              /* of the 8-bit states' rounding */
} strata_adamw_desc;

strata_status strata_adamw(const strata_adamw_desc* desc, const strata_params* params, void* m, void* v,
                           uint8_t* m_scales, uint8_t* v_scales, const float* factor, void* stream);

/* The values of 8-bit states (second: v), exact in bf16 too: x [n] of dtype, 1 <= n < 2^32. */
strata_status strata_adamw_unpack(const uint8_t* codes, const uint8_t* scales, int64_t n, int32_t second, void* x,
                                  strata_dtype dtype, void* stream);

/* ---- a8: tile stitch S = D^-1 P^T W (App. F, Eq. stitch) -------------------
 * Regular tiling: tile t = a*ntx + b has origin (a*stride_y, b*stride_x) on the
 * face.  tiles: [nty*ntx, P, Ht, Wt, C] of dtype; window: float32 [Ht*Wt],
 * >= 0; out: [P, Hf, Wf, C] of dtype.  For every face cell:
 *   out = (sum_t w_t * value_t) / (sum_t w_t)  over the tiles t covering it,
 * summed in ascending a, then b, with fused multiply-adds from zero, divided
 * with correct rounding; bf16 data accumulate in float32, f32 data in float64.
 * Cells no tile weights (sum 0) are written as 0.  Requires
 * (nty-1)*stride_y + Ht <= Hf and (ntx-1)*stride_x + Wt <= Wf.  Bit-exact. */
strata_status strata_tile_blend(const void* tiles, int32_t nty, int32_t ntx, int32_t P,
                                int32_t Ht, int32_t Wt, int32_t C, int32_t stride_y,
                                int32_t stride_x, const float* window, void* out, int32_t Hf,
                                int32_t Wf, strata_dtype dtype, void* stream);

/* ---- a4-a6 + a8: face step with the stitch fused into the forward ----------
 * (Sec. 3.2 attention on each tile of one face, App. F, Eq. stitch.)  The
 * batch of `desc` is the nty x ntx tiling of one face, tile t = a*ntx + b at
 * origin (a*stride_y, b*stride_x), P = heads*Z planes, Ht = H, Wt = W,
 * C = head_dim, window float32 [H*W] >= 0, face [heads*Z, Hf, Wf, head_dim]
 * of the problem's dtype.  Two calls on one stream give
 *   strata_tile_blend(strata_na3d_fwd_ex(...))      bit for bit:
 * strata_na3d_fwd_stitch, then strata_tile_blend_overlap with the same tiles,
 * tiling, window and face.  The first writes the attention output (options
 * and lse as in strata_na3d_fwd_ex) and stores every cell that one tile alone
 * covers straight into `face`, computed as the stitch computes it: the tile's
 * value fma(w, v, +0) / w rounded to the dtype, which for 2^-8 <= w <= 1 (the
 * linear ramp's range) is v itself with -0 turned into +0, and 0 where w = 0.  The other cells go to `tiles`
 * ([B, heads, Z, H, W, head_dim], caller-owned scratch; the contents of
 * single-cover cells are unspecified).  The second stitches the cells that two
 * or more tiles cover and leaves the rest of the face as it is.  The fusion
 * applies to bf16 tilings whose tiles cover the face with
 * stride <= extent <= 2 stride on both axes, at the shape of the level-sweep
 * forward (3x7x7, Z = 8, head_dim 64); elsewhere the first call writes every
 * tile output and stitches the whole face, and the second re-stitches cells
 * with the same values.  tiles, face and the inputs must not overlap.
 * Validation as strata_na3d_fwd_ex and strata_tile_blend, plus B = nty*ntx.
 * One or two kernel launches per call; nothing is allocated. */
strata_status strata_na3d_fwd_stitch(const strata_na3d_desc* desc, const strata_na3d_opts* opts,
                                     const void* q, const void* k, const void* v, const float* cs,
                                     void* tiles, float* lse, int32_t nty, int32_t ntx,
                                     int32_t stride_y, int32_t stride_x, const float* window,
                                     void* face, int32_t Hf, int32_t Wf, void* stream);
strata_status strata_tile_blend_overlap(const void* tiles, int32_t nty, int32_t ntx, int32_t P,
                                        int32_t Ht, int32_t Wt, int32_t C, int32_t stride_y,
                                        int32_t stride_x, const float* window, void* out,
                                        int32_t Hf, int32_t Wf, strata_dtype dtype, void* stream);

/* ---- Duo-grid halo padding P (App. F, "DUO-style boundary padding") --------
 * faces: [6, P, n, n, C] of dtype (P planes of n x n cells with C channels per
 * face, orientation as in strata_stereo_coords); padded: [6, P, n + 2 halo,
 * n + 2 halo, C].  Interior cells are copied.  Halo cell (i, j) of face f
 * (i or j outside [0, n)) extends f's equiangular mesh on f's own plane
 * (angles -pi/4 + (index + 1/2)(pi/2)/n), is projected to the sphere, and
 * takes the inverse great-circle-distance weighted average of the 4 cells
 * nearest to that point on the face containing it (the face of its largest
 * coordinate; a point on an edge or corner, where face scores are equal on a
 * 1e-12 grid, belongs to the lowest-numbered face); distances equal on a
 * 1e-12-radian grid are ordered by (row, column), a cell at distance 0 takes
 * the whole weight.  Sums nearest first, in float32 for bf16 data, float64 for
 * float32 data.  Both buffers are device memory owned by the caller and must
 * not overlap.  n >= 16, 1 <= halo <= n/4, 6 P n rows plus one block per 256
 * halo cells below 2^31; otherwise STRATA_ERR_INVALID_ARG and nothing is
 * launched.  One kernel launch on `stream`. */
strata_status strata_duo_pad(const void* faces, int32_t P, int32_t n, int32_t C, int32_t halo, void* padded,
                             strata_dtype dtype, void* stream);

/* The same padding operator P built once and applied many times (App. F: P is a
 * fixed sparse matrix with 4 non-zeros per halo cell, so a model that pads
 * every layer of a rollout reuses it), and its transpose for gradients.
 *
 * strata_duo_plan_bytes: size of the plan for (n, halo), 0 if the pair is
 * invalid or too large (n + 2 halo < 2^14, 4 entries per halo cell below
 * 2^31).  strata_duo_plan: writes the plan (geometry only, no field
 * data: P and its transpose) into `plan`, caller-owned device memory of at
 * least that many bytes, 16-byte aligned; its contents are opaque and valid
 * for this (n, halo) only.  The build is deterministic.
 * strata_duo_pad_planned: as strata_duo_pad, with the neighbours and weights
 * read from a plan written by strata_duo_plan for the same (n, halo); results
 * are identical to strata_duo_pad's.
 * strata_duo_pad_vjp: the adjoint, grad_faces = P^T grad_padded
 * (grad_padded: [6, P, n + 2 halo, n + 2 halo, C], grad_faces: [6, P, n, n,
 * C], both of dtype, not overlapping): every face cell's interior gradient
 * plus, for each halo cell whose 4 neighbours include it, that halo cell's
 * gradient times the weight, summed in ascending padded-cell order (face,
 * row, column) after the interior term, with fused multiply-adds; float32
 * sums for bf16 data, float64 for float32 data; one rounding.  Deterministic.
 * P <= 65535.
 * Errors: STRATA_ERR_INVALID_ARG for the rules of strata_duo_pad, a NULL or
 * misaligned plan, or plan_bytes below strata_duo_plan_bytes(n, halo); nothing
 * is launched then. */
size_t strata_duo_plan_bytes(int32_t n, int32_t halo);
strata_status strata_duo_plan(int32_t n, int32_t halo, void* plan, size_t plan_bytes, void* stream);
strata_status strata_duo_pad_planned(const void* faces, int32_t P, int32_t n, int32_t C, int32_t halo,
                                     const void* plan, size_t plan_bytes, void* padded, strata_dtype dtype,
                                     void* stream);
strata_status strata_duo_pad_vjp(const void* grad_padded, int32_t P, int32_t n, int32_t C, int32_t halo,
                                 const void* plan, size_t plan_bytes, void* grad_faces, strata_dtype dtype,
                                 void* stream);

/* ---- a8: Kaiser-Bessel-derived blend window (App. F, "Tile stitching") -----
 * window[y * Wt + x] = w(y, Ht) * w(x, Wt) (float32 [Ht * Wt], device) with,
 * per axis of length L, w(i) = 1 in the interior and, over the `overlap` cells
 * at each end, the rising half of the KBD window of length 2*overlap:
 *   w(i) = sqrt(sum_{j<=i} k_j / sum_{j<=overlap} k_j),
 *   k_j = I0(beta sqrt(1 - (2j/overlap - 1)^2)),  j = 0..overlap,
 * mirrored at the far end (the smaller value where both ends reach).  The
 * paper gives no alpha or taper length: beta (= pi alpha) is an argument and
 * the taper spans the overlap, as the linear ramp does.  1 <= overlap <=
 * min(Ht, Wt); 0 <= beta <= 700.  Computed in float64, rounded once. */
strata_status strata_kbd_window(int32_t Ht, int32_t Wt, int32_t overlap, double beta, float* window,
                                void* stream);

/* ---- a8': tile extraction P (App. F) ---------------------------------------
 * tiles[t, p, i, j, c] = face[p, a*stride_y + i, b*stride_x + j, c] (exact copy). */
strata_status strata_tile_extract(const void* face, int32_t nty, int32_t ntx, int32_t P,
                                  int32_t Ht, int32_t Wt, int32_t C, int32_t stride_y,
                                  int32_t stride_x, int32_t Hf, int32_t Wf, void* tiles,
                                  strata_dtype dtype, void* stream);

/* ---- a3: window indexing of one axis (Sec. 3.2, NATTEN's border-clamped ----
 * neighbourhood; bit-exact integer export).  For an axis of extent L and
 * window k (odd with 1 <= k <= L, or k == L): starts[i] = min(max(i - (k-1)/2,
 * 0), L - k) is the first position of query i's window [starts[i],
 * starts[i] + k); [qlo[j], qhi[j]] is the contiguous range of queries whose
 * window holds position j.  starts, qlo, qhi: device int32[L] each, written by
 * one launch on `stream`; STRATA_ERR_INVALID_ARG for other (L, k) or a NULL /
 * misaligned pointer, with nothing launched. */
strata_status strata_na_axis_index(int32_t L, int32_t k, int32_t* starts, int32_t* qlo,
                                   int32_t* qhi, void* stream);

/* ---- status ---------------------------------------------------------------- */
const char* strata_status_string(strata_status status);
/* Detail of the last non-OK status returned on the calling thread ("" if none). */
const char* strata_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* STRATA_H_ */
