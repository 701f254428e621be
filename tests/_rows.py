"""Problems of projection rows for the GPU tests: seeded inputs whose float64 copies
the oracle takes, guarded output buffers, and the tolerances.

A tolerance is one rounding to the output's type, eps/2 of the value (bf16 2^-8,
fp32 2^-24), plus the float32 arithmetic before it.  That is relative to the
magnitudes that are added (a rotated pair's, a sum's terms): the mean of d squares
is 8 sequential additions and a tree of at most 4 levels (12 2^-24), its root and
reciprocal at most 3 2^-24, then at most 8 more roundings: below 2^-19.  A sum of up
to 16 shared heads adds 16 2^-24, within the same 2^-19.  A weight gradient is a sum
of at most a few hundred sequential additions of such terms (2^-24 each): 2^-15.
"""
import dataclasses

import numpy as np
import torch

from oracle import rows as R
from paper_2606_31248_amd import binding as B

ARITH, WEIGHT_SUM = 2.0 ** -19, 2.0 ** -15
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


@dataclasses.dataclass
class Case:
    dtype: str
    B: int
    heads: int
    kv: int
    Z: int
    H: int
    W: int
    d: int
    gate: int = 0
    pad: int = 0
    rope: bool = True
    norm: bool = True
    weights: bool = True

    @property
    def p(self):
        return R.Rows(self.heads, self.kv, self.d, self.gate, self.norm)

    @property
    def grid(self):
        return (self.B, self.Z, self.H, self.W)

    @property
    def shape(self):
        return (self.B, self.heads, self.Z, self.H, self.W, self.d)

    def gate_shape(self):
        return self.shape if self.gate > 1 else self.shape[:-1]

    def desc(self):
        return B.make_qkv_desc(self.B, self.heads, self.Z, self.H, self.W, self.d,
                               B.STRATA_BF16 if self.dtype == "bf16" else B.STRATA_F32, kv_heads=self.kv,
                               gate_dim=self.gate, row_stride=(self.p.width + self.pad + 7) // 8 * 8, qk_norm=self.norm)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, dtype, g, mult=1.0):
    """On the GPU in `dtype`; the values are made on the host, so they do not depend on the device."""
    return (torch.randn(shape, generator=g) * mult).to(TYPE[dtype]).cuda()


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def guarded(shape, dtype, fill=7.0):
    """A tensor inside a larger buffer: (tensor, check), check() asserting that nothing behind it was written."""
    n = int(np.prod(shape))
    buf = torch.full((n + 512,), fill, dtype=dtype, device="cuda")

    def check():
        assert bool((buf[n:] == fill).all()), "written behind the tensor"
    return buf[:n].view(shape), check


def phases(c: Case, g):
    th = (torch.rand((c.B, c.H, c.W, c.d // 2), generator=g, dtype=torch.float64) * 2 - 1) * 200
    return torch.stack([th.cos(), th.sin()], -1).float().cuda()


class Problem:
    """Inputs and guarded outputs of one case."""

    def __init__(self, c: Case, seed=0):
        g = gen(seed + 1000)
        t = TYPE[c.dtype]
        self.c, self.desc = c, c.desc()
        self.rows = normal(c.grid + (self.desc.row_stride,), c.dtype, g)
        self.rows *= torch.exp(torch.randn(self.desc.row_stride, generator=g)).to(t).cuda()
        self.cs = phases(c, g) if c.rope else None
        self.wq, self.wk = ((1 + 0.3 * torch.randn(c.d, generator=g)).cuda() for _ in range(2)) if c.weights else (None, None)
        self.up = {n: normal(c.shape, c.dtype, g) for n in ("dq", "dk", "dv")}
        self.up["dgate"] = normal(c.gate_shape(), c.dtype, g) if c.gate else None
        self.checks = []

    def new(self, shape, dtype, fill=7.0):
        x, check = guarded(shape, dtype, fill)
        self.checks.append(check)
        return x

    def heads_out(self, with_gate=True):
        t = TYPE[self.c.dtype]
        out = {n: self.new(self.c.shape, t) for n in ("q", "k", "v")}
        out["gate"] = self.new(self.c.gate_shape(), t) if self.c.gate and with_gate else None
        return out

    def codes_out(self):
        return self.new(self.c.grid + (self.desc.kept,), torch.int8, 77), \
            self.new(self.c.grid + (self.desc.kept // 32,), torch.uint8, 77)

    def forward(self, codes=None, scales=None):
        o = self.heads_out()
        B.strata_qkv_heads(self.desc, self.rows, self.wq, self.wk, self.cs, o["q"], o["k"], o["v"], o["gate"], codes, scales)
        return o

    def again(self, codes, scales):
        o = self.heads_out(self.c.gate > 1)
        B.strata_qkv_heads_ckpt(self.desc, codes, scales, self.wq, self.wk, self.cs, o["q"], o["k"], o["v"], o["gate"])
        return o

    def backward(self, rows=None, codes=None, scales=None):
        t = TYPE[self.c.dtype]
        drows = self.new(self.c.grid + (self.desc.row_stride,), t)
        dwq, dwk = (self.new((self.c.d,), torch.float32) if self.c.weights else None for _ in range(2))
        ws = self.new((B.strata_qkv_heads_bwd_workspace_size(self.desc),), torch.uint8, 77)
        B.strata_qkv_heads_bwd(self.desc, rows, codes, scales, self.wq, self.wk, self.cs, self.up["dq"], self.up["dk"],
                               self.up["dv"], self.up["dgate"], drows, dwq, dwk, ws)
        return dict(drows=drows, dwq=dwq, dwk=dwk)

    def rows64(self):
        return f64(self.rows)[..., :self.c.p.width]

    def check_guards(self):
        torch.cuda.synchronize()
        for check in self.checks:
            check()

    def want_forward(self, rows64):
        return R.forward(self.c.p, rows64, f64(self.wq), f64(self.wk), f64(self.cs))

    def want_backward(self, rows64):
        return R.backward(self.c.p, rows64, wq=f64(self.wq), wk=f64(self.wk), cs=f64(self.cs),
                          **{n: f64(x) for n, x in self.up.items()})


def check_heads(got, want, dtype, what):
    """q and k: one rounding and the arithmetic, relative to the pair's length; the rest is copied."""
    for n in want:
        g = f64(got[n])
        if n in ("v", "gate"):
            assert np.array_equal(g, want[n]), f"{what}: {n} differs"
            continue
        pair = np.repeat(np.abs(want[n][..., 0::2]) + np.abs(want[n][..., 1::2]), 2, axis=-1)
        tol = HALF_STEP[dtype] * np.abs(want[n]) * (1 + ARITH) + 2 * ARITH * pair
        worst = np.max(np.abs(g - want[n]) - tol)
        assert worst <= 0, f"{what}: {n} off by {worst:.3e} more than its tolerance"


def check_grads(got, want, dtype, what):
    g = f64(got["drows"])[..., :want["drows"].shape[-1]]
    tol = HALF_STEP[dtype] * np.abs(want["drows"]) + 2 * ARITH * want["mag_drows"]
    worst = np.max(np.abs(g - want["drows"]) - tol)
    assert worst <= 0, f"{what}: drows off by {worst:.3e} more than its tolerance"
    for n in ("dwq", "dwk"):
        if n in want:
            worst = np.max(np.abs(f64(got[n]) - want[n]) - WEIGHT_SUM * want["mag_" + n])
            assert worst <= 0, f"{what}: {n} off by {worst:.3e} more than its tolerance"
