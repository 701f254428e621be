"""The hot path on device tensors, as sequences of libstrata calls.

One rollout pass: coordinates (Eq. 1) -> StereoRoPE phases -> neighbourhood
attention forward with the rotation fused into the Q/K loads -> tile stitch
S = D^-1 P^T W.  One training block, from its projection's rows to their gradient:
``block_forward`` and ``block_backward``, with the rows and the attention's output
kept between them as they are or in 8 bits.
PyTorch only allocates device memory and supplies the stream.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from . import binding as B

ROPE_BASE = 100.0


@dataclasses.dataclass
class TileGeometry:
    face: torch.Tensor   # int32 [B] on device
    oy: torch.Tensor     # int32 [B] token row of the tile origin
    ox: torch.Tensor     # int32 [B] token column of the tile origin
    face_cells: int = 2048
    patch: int = 4


def stereo_phases(geom: TileGeometry, H: int, W: int, head_dim: int,
                  coords: Optional[torch.Tensor] = None, cs: Optional[torch.Tensor] = None,
                  base: float = ROPE_BASE):
    """Coordinates [B, H, W, 2] and phase table [B, H, W, head_dim/2, 2] (float32)."""
    Bt = geom.face.shape[0]
    dev = geom.face.device
    if coords is None:
        coords = torch.empty((Bt, H, W, 2), dtype=torch.float32, device=dev)
    if cs is None:
        cs = torch.empty((Bt, H, W, head_dim // 2, 2), dtype=torch.float32, device=dev)
    B.strata_stereo_coords(geom.face, geom.oy, geom.ox, H, W, geom.face_cells, geom.patch,
                           0.0, coords)  # 0: the library's Eq. 1 length for these faces
    B.strata_stereorope_phases(coords, head_dim, base, cs)
    return coords, cs


def na3d_forward(q, k, v, window, scale, cs=None, out=None, lse=None):
    if out is None:
        out = torch.empty_like(q)
    desc = B.desc_for(q, window, scale)
    B.strata_na3d_fwd(desc, q, k, v, cs, out, lse)
    return out


# what the attention's lse and output depend on, of a BlockSaved
_OF_THE_FORWARD = frozenset(("qkv", "window", "scale", "wq", "wk", "cs", "rows"))


@dataclasses.dataclass
class BlockSaved:
    """What a block keeps: the rows and the attention's output, each as it was or as (codes, scales), the
    softmax's lse and, with a gate logit per head, the gate.

    out and lse are the forward's.  `again`: they are not those of the values that block_backward works on (rows
    in 8 bits, or a field that shapes the attention assigned since), and it runs the attention once more for its own;
    out is then for the caller, whose projection behind the block takes its weights' gradient from it.  A state that
    the caller constructs (dataclasses.replace does) is taken to hold the lse and out of its rows unless it says again."""
    qkv: B.QKVDesc
    window: tuple
    scale: float
    wq: Optional[torch.Tensor]
    wk: Optional[torch.Tensor]
    cs: Optional[torch.Tensor]
    lse: torch.Tensor
    rows: object
    out: object
    gate: Optional[torch.Tensor] = None
    again: bool = False

    def __setattr__(self, name, value):
        if name in _OF_THE_FORWARD and "again" in self.__dict__:  # the last field: not while it is being made
            self.__dict__["again"] = True
        super().__setattr__(name, value)

    def nbytes(self) -> int:
        """Bytes kept for this block, besides the weights and the phases that all blocks share."""
        held = [self.lse, self.gate]
        for x in (self.rows, self.out):
            held += list(x) if isinstance(x, tuple) else [x]
        return sum(t.numel() * t.element_size() for t in held if t is not None)


def _heads_like(d: B.QKVDesc, rows_dtype, device):
    """Uninitialised q, k, v and gate (None without one) of a block."""
    shape = (d.B, d.heads, d.Z, d.H, d.W, d.head_dim)
    new = lambda s: torch.empty(s, dtype=rows_dtype, device=device)  # noqa: E731
    return new(shape), new(shape), new(shape), new(shape if d.gate_dim > 1 else shape[:-1]) if d.gate_dim else None


def _attention_of(d: B.QKVDesc, window, scale, gate):
    """Descriptor and options of the block's attention: norm and rotation are already in q and k."""
    desc = B.make_desc(d.B, d.heads, d.Z, d.H, d.W, d.head_dim, window, scale, d.dtype)
    return desc, B.make_opts(gate=gate) if gate is not None else None


def block_forward(rows, qkv: B.QKVDesc, window, scale, wq=None, wk=None, cs=None, eight_bit: bool = False):
    """Attention of one block from its projection's rows [B, Z, H, W, row_stride]: (out, saved).

    out: [B, heads, Z, H, W, head_dim], gated by the rows' gate logits if there are any.  eight_bit: `saved`
    holds the rows and out in 8 bits (just over half the bytes of bf16) instead of the tensors themselves, and
    block_backward runs the attention's forward once more.  Its gradient is then off by about 2 % at logits of
    order one and by more as they grow (13 % at a deviation of 16)."""
    q, k, v, gate = _heads_like(qkv, rows.dtype, rows.device)
    kept = rows
    codes = scales = None
    if eight_bit:
        grid = (qkv.B, qkv.Z, qkv.H, qkv.W)
        codes = torch.empty(grid + (qkv.kept,), dtype=torch.int8, device=rows.device)
        scales = torch.empty(grid + (qkv.kept // 32,), dtype=torch.uint8, device=rows.device)
        kept = (codes, scales)
    B.strata_qkv_heads(qkv, rows, wq, wk, cs, q, k, v, gate, codes, scales)
    desc, opts = _attention_of(qkv, window, scale, gate)
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device)
    B.strata_na3d_fwd_ex(desc, opts, q, k, v, None, out, lse)
    held = out
    if eight_bit:
        held = (torch.empty(out.numel(), dtype=torch.int8, device=out.device),
                torch.empty((out.numel() + 31) // 32, dtype=torch.uint8, device=out.device))
        B.strata_ckpt_pack(out, *held)
    return out, BlockSaved(qkv, tuple(window), scale, wq, wk, cs, lse, kept, held,
                           gate if qkv.gate_dim == 1 else None, again=eight_bit)


def block_backward(saved: BlockSaved, dout):
    """Gradient of block_forward's out: (drows [B, Z, H, W, row_stride], dwq, dwk), zeros behind the rows' width.

    From 8 bits they are the gradients at the values that the codes stand for: the attention's forward is run
    again on these, since weights exp(s - lse) with the lse of the values before would not sum to 1 (and exceed the
    range that the attention's backward has for them)."""
    d = saved.qkv
    q, k, v, gate = _heads_like(d, dout.dtype, dout.device)
    rows, codes, scales = (None, *saved.rows) if isinstance(saved.rows, tuple) else (saved.rows, None, None)
    if codes is not None:
        B.strata_qkv_heads_ckpt(d, codes, scales, saved.wq, saved.wk, saved.cs, q, k, v,
                                gate if d.gate_dim > 1 else None)
        gate = saved.gate if d.gate_dim == 1 else gate
    else:
        B.strata_qkv_heads(d, rows, saved.wq, saved.wk, saved.cs, q, k, v, gate)
    desc, opts = _attention_of(d, saved.window, saved.scale, gate)
    out, lse = saved.out, saved.lse
    if saved.again:
        out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device)
        B.strata_na3d_fwd_ex(desc, opts, q, k, v, None, out, lse)
    dq, dk, dv = (torch.empty_like(q) for _ in range(3))
    dgate = None if gate is None else torch.empty_like(gate)
    ws = torch.empty(B.strata_na3d_bwd_ex_workspace_size(desc, opts), dtype=torch.uint8, device=q.device)
    B.strata_na3d_bwd_ex(desc, opts, q, k, v, None, out, dout, lse, dq, dk, dv, dgate, ws)
    drows = torch.empty((d.B, d.Z, d.H, d.W, d.row_stride), dtype=dout.dtype, device=dout.device)
    if d.row_stride > d.width:
        drows[..., d.width:] = 0
    dwq, dwk = (None if w is None else torch.empty_like(w) for w in (saved.wq, saved.wk))
    ws = torch.empty(B.strata_qkv_heads_bwd_workspace_size(d), dtype=torch.uint8, device=q.device)
    B.strata_qkv_heads_bwd(d, rows, codes, scales, saved.wq, saved.wk, saved.cs, dq, dk, dv, dgate, drows, dwq, dwk,
                           ws)
    return drows, dwq, dwk


def face_step(q, k, v, geom: TileGeometry, window, scale, tiling, blend_window, face_out,
              coords=None, cs=None, out=None, fused: bool = True, opts=None):
    """One face rollout step: per-tile NA3D forward with StereoRoPE, then the stitch.

    q, k, v: [T, heads, Z, Ht, Wt, d]; tiling = (nty, ntx, stride_y, stride_x);
    the tile outputs are viewed as [T, heads*Z, Ht, Wt, d] planes for the blend;
    face_out: [heads*Z, Hf, Wf, d].  fused: the forward stores the cells one tile
    alone covers straight into the face and the stitch visits only the overlaps
    (the same face bit for bit); `out` then holds only the overlap cells."""
    T, heads, Z, Ht, Wt, d = q.shape
    coords, cs = stereo_phases(geom, Ht, Wt, d, coords, cs)
    if out is None:
        out = torch.empty_like(q)
    nty, ntx, sy, sx = tiling
    planes = out.view(T, heads * Z, Ht, Wt, d)
    desc = B.desc_for(q, window, scale)
    if fused:
        B.strata_na3d_fwd_stitch(desc, opts, q, k, v, cs, out, None, nty, ntx, sy, sx, blend_window, face_out)
        B.strata_tile_blend_overlap(planes, nty, ntx, sy, sx, blend_window, face_out)
    else:
        B.strata_na3d_fwd_ex(desc, opts, q, k, v, cs, out, None)
        B.strata_tile_blend(planes, nty, ntx, sy, sx, blend_window, face_out)
    return face_out
