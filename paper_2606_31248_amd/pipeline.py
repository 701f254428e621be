"""The hot path on device tensors, as sequences of libstrata calls.

One rollout pass: coordinates (Eq. 1) -> StereoRoPE phases -> neighbourhood
attention forward with the rotation fused into the Q/K loads -> tile stitch
S = D^-1 P^T W.  One training block, from its projection's rows to their gradient:
``block_forward`` and ``block_backward``, with the rows and the attention's output
kept between them as they are or in 8 bits.  Around the blocks: the residual stream's
addition with its norm (``norm_forward``, ``norm_backward``), and the update of all weights
from their gradients (``AdamW``).
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


@dataclasses.dataclass
class NormSaved:
    """What the entry of a block keeps: the stream (res itself without a branch), the branch that was added where it
    has a gate, the vectors, and the norm's output, as it is or as (codes, scales), for the weights' gradient of the
    projection that read it."""
    desc: B.NormDesc
    total: torch.Tensor
    x: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]
    shift: Optional[torch.Tensor]
    held: object

    def output(self) -> torch.Tensor:
        """The norm's output, from 8 bits the values of its codes."""
        if not isinstance(self.held, tuple):
            return self.held
        y = torch.empty_like(self.total)
        B.strata_ckpt_unpack(*self.held, y)
        return y


def norm_forward(res, x=None, gate=None, scale=None, shift=None, group_rows: Optional[int] = None, eps: float = 1e-6,
                 eight_bit: bool = False):
    """Entry of a block: (y, sum, saved), sum = res + gate x (res itself without x) and y = scale rms(sum) + shift.

    res, x: [..., width]; gate, scale, shift: float32 [groups, width] or None, one for every group_rows consecutive
    rows (default: one for all).  eight_bit: `saved` holds y in 8 bits, for a width of whole 32."""
    desc = B.make_norm_desc(res, group_rows, eps)
    total = res if x is None else torch.empty_like(res)
    y = torch.empty_like(res)
    codes = scales = None
    if eight_bit:
        codes = torch.empty(res.shape, dtype=torch.int8, device=res.device)
        scales = torch.empty(res.shape[:-1] + (res.shape[-1] // 32,), dtype=torch.uint8, device=res.device)
    B.strata_residual_norm(desc, x, gate, res, scale, shift, None if x is None else total, y, codes, scales)
    return y, total, NormSaved(desc, total, None if gate is None else x, gate, scale, shift, (codes, scales) if eight_bit else y)


def norm_backward(saved: NormSaved, dy, dsum=None):
    """Gradients of norm_forward for those of y and of sum (None: 0): (dres, dx, dgate, dscale, dshift).

    dx is dres itself without a gate; None for a vector that was None."""
    dres = torch.empty_like(dy)
    dx, dgate = (None, None) if saved.gate is None else (torch.empty_like(dy), torch.empty_like(saved.gate))
    dscale, dshift = (None if v is None else torch.empty_like(v) for v in (saved.scale, saved.shift))
    ws = torch.empty(B.strata_residual_norm_bwd_workspace_size(saved.desc), dtype=torch.uint8, device=dy.device)
    B.strata_residual_norm_bwd(saved.desc, saved.total, saved.x, saved.gate, saved.scale, dy, dsum, dres, dx, dgate, dscale,
                               dshift, ws)
    return dres, dres if dx is None else dx, dgate, dscale, dshift


def _current_stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


class AdamW:
    """AdamW over a list of weights, with the norm of their gradients clipped and the states in 32 bits or in 8.

    p, g, copies: as binding.make_params takes them; the list keeps the tensors alive and takes them to stay where they
    are.  Gradients that are allocated anew, as where zero_grad sets them to None, are given to `renew` before the step
    that takes them: a list of weights' own .grad refuses a step on one that was replaced.  m, v and, in 8 bits, m_scales
    and v_scales are the states, flat, and `steps` the steps taken: what a checkpoint stores.  A step whose gradients
    are not all finite changes no tensor if it clips (max_norm, which may be infinity), but is counted.  A captured step
    repeats its learning rate, its number and its seed."""

    def __init__(self, p, g, copies=None, eight_bit: bool = False, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, weight_decay: float = 0.0, max_norm: Optional[float] = None, seed: int = 0):
        self._captured = []
        self._take(p, g, copies)
        self.hyper = dict(beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay)
        self.max_norm, self.seed, self.steps = max_norm, seed, 0
        n, dev = self.params.places, self.params.device
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8 if eight_bit else torch.float32, device=dev) for _ in range(2))
        self.m_scales, self.v_scales = ((torch.zeros(n // 32, dtype=torch.uint8, device=dev) for _ in range(2)) if eight_bit
                                        else (None, None))
        self._norm = torch.empty(2, dtype=torch.float32, device=dev)

    def _take(self, p, g, copies):
        params = B.make_params(p, g, copies)
        ws = torch.empty(B.strata_grad_norm_workspace_size(params), dtype=torch.uint8, device=params.device)
        self.params, self._ws = params, ws
        self._stream, self._others = _current_stream(params.device), {}  # of the list, and of steps elsewhere
        self._own = [(w, d) for w, d in zip(*params.tensors[:2]) if d is not None and w.is_leaf and w.grad is d]

    def renew(self, g, copies=None):
        """Other gradients (None: that tensor is left as it is) and copies (default: the present ones) from the next step
        on; weights, states and steps stay.  Makes the list's table and copies it to the device, 0.4 ms for 300 tensors:
        gradients that stay where they are (zero_grad(set_to_none=False)) need none of it."""
        p, *old = self.params.tensors
        others = self._others.values()
        self._take(p, g, old[1] if copies is None else copies)
        for s in others:  # let go once these streams have read them
            for t in old[0] + old[1]:
                if t is not None:
                    t.record_stream(s)

    def step(self, lr: float) -> Optional[torch.Tensor]:
        """One step from the gradients that are in place.  With max_norm: float32 [2] on the device, the gradients'
        norm and the factor they were multiplied by, overwritten by the next step."""
        for w, d in self._own:
            if w.grad is not d:
                raise ValueError("AdamW: a listed gradient is no longer its weight's .grad; renew() takes the new ones")
        norm, k = None, self.steps + 1
        if self.max_norm is not None:
            norm = self._norm
            B.strata_grad_norm(self.params, self.max_norm, norm, self._ws)
        desc = B.make_adamw_desc(lr, k, seed=(self.seed << 40) + k, **self.hyper)
        B.strata_adamw(desc, self.params, self.m, self.v, self.m_scales, self.v_scales, None if norm is None else norm[1:])
        self.steps = k   # a step that was refused is none
        # a list that renew replaces is let go, but not under a graph, nor before another stream's kernels have read it
        if torch.cuda.is_current_stream_capturing():
            if not self._captured or self._captured[-1][0] is not self.params:
                self._captured.append((self.params, self._ws))
            return norm
        stream = B._on_gpu(self.params.index, None)
        if stream != self._stream:
            s = self._others[stream] = torch.cuda.current_stream(self.params.device)
            for t in (self.params.table, self._ws):
                t.record_stream(s)
        return norm

    def moments(self, i: int):
        """(m, v) of tensor i as float32 tensors of its shape."""
        w = self.params.tensors[0][i]
        at, n = self.params.at[i], w.numel()
        cut = lambda t, k=1: t[at // k:at // k + -(-n // k)]  # noqa: E731
        if self.m_scales is None:
            return cut(self.m).clone().view(w.shape), cut(self.v).clone().view(w.shape)
        m, v = (torch.empty(w.shape, dtype=torch.float32, device=w.device) for _ in range(2))
        if n:
            B.strata_adamw_unpack(cut(self.m), cut(self.m_scales, 32).clone(), m, second=False)
            B.strata_adamw_unpack(cut(self.v), cut(self.v_scales, 32).clone(), v, second=True)
        return m, v


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
