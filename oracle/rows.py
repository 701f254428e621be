"""Oracle: projection rows and the attention's head layout, and activations held in
8 bits (test infrastructure, CPU only, numpy float64).

A row is [q | k | v | gate] with the head before its channels.  `Rows` names the
sizes; every function takes and returns float64 arrays, rows [B, Z, H, W, width],
heads [B, heads, Z, H, W, d].
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import numpy as np


@dataclasses.dataclass
class Rows:
    heads: int
    kv: int
    d: int
    gate: int = 0          # logits per head: 0, 1 or d
    norm: bool = True
    eps: float = 1e-6

    @property
    def kept(self):
        return (self.heads + 2 * self.kv + (self.heads if self.gate > 1 else 0)) * self.d

    @property
    def width(self):
        return self.kept + (self.heads if self.gate == 1 else 0)


# ---- 8 bits -----------------------------------------------------------------------

def encode(x):
    """Flat float64 values -> (codes int8, exponents uint8), group by group of 32."""
    x = np.asarray(x, dtype=np.float64).reshape(-1)
    v = np.pad(x, (0, -x.size % 32)).reshape(-1, 32)
    fine = np.isfinite(v).all(1)
    v = np.where(fine[:, None], v, 0.0)
    top = np.abs(v).max(1)
    s = np.where(top > 0, np.frexp(top)[1] + 126, 0)  # top = m 2^e, 1/2 <= m < 1: 64 to 128 steps of 2^(e - 7)
    s = np.where(np.rint(np.ldexp(top, 133 - s)) > 127, s + 1, s)
    s = np.clip(s, 7, 254)
    codes = np.clip(np.rint(np.ldexp(v, 133 - s[:, None])), -127, 127).astype(np.int8)
    return codes.reshape(-1)[:x.size], np.where(fine, s, 255).astype(np.uint8)


def decode(codes, scales):
    """The values of flat codes and exponents (NaN where the exponent is 255)."""
    s = np.repeat(np.asarray(scales, np.int64), 32)[:codes.size]
    return np.where(s == 255, np.nan, codes.astype(np.float64) * 2.0 ** (s - 133.0))


# ---- rows -> heads ----------------------------------------------------------------

def _heads_of(x, heads, d):
    """[B, Z, H, W, heads * d] -> [B, heads, Z, H, W, d]."""
    return np.moveaxis(x.reshape(x.shape[:-1] + (heads, d)), 4, 1)


def _rows_of(x):
    """[B, heads, Z, H, W, d] -> [B, Z, H, W, heads * d]."""
    y = np.moveaxis(x, 1, 4)
    return y.reshape(y.shape[:4] + (-1,))


def split(p: Rows, rows):
    """q [B, heads, ...], k, v [B, kv, ...] and the gate [B, heads, ...(, d)] or None, as they stand in the rows."""
    a, b = p.heads * p.d, p.kv * p.d
    q, k, v, g = np.split(rows[..., :p.width], [a, a + b, a + 2 * b], axis=-1)
    gate = None
    if p.gate == 1:
        gate = np.moveaxis(g, 4, 1)
    elif p.gate:
        gate = _heads_of(g, p.heads, p.d)
    return _heads_of(q, p.heads, p.d), _heads_of(k, p.kv, p.d), _heads_of(v, p.kv, p.d), gate


def turn(x, cs, back=False):
    """Rotate channel pairs by the phase table [B, H, W, d/2, 2]."""
    if cs is None:
        return x
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * (cs[..., 0] + (-1j if back else 1j) * cs[..., 1])[:, None, None]
    out = np.empty(x.shape)
    out[..., 0::2], out[..., 1::2] = z.real, z.imag
    return out


def rms(p: Rows, x):
    """x over its root mean square, and 1 / that root."""
    if not p.norm:
        return x, np.ones(x.shape[:-1] + (1,))
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + p.eps)
    return x * r, r


def forward(p: Rows, rows, wq=None, wk=None, cs=None):
    """dict(q, k, v, gate) in the head layout."""
    q, k, v, gate = split(p, rows)
    n = p.heads // p.kv
    out = dict(q=turn(rms(p, q)[0] * (1.0 if wq is None else wq), cs),
               k=np.repeat(turn(rms(p, k)[0] * (1.0 if wk is None else wk), cs), n, axis=1),
               v=np.repeat(v, n, axis=1))
    if gate is not None:
        out["gate"] = gate
    return out


def _shared(p: Rows, x):
    """Sum over the query heads of each key head."""
    return x.reshape((x.shape[0], p.kv, p.heads // p.kv) + x.shape[2:]).sum(2)


def backward(p: Rows, rows, dq, dk, dv, dgate=None, wq=None, wk=None, cs: Optional[np.ndarray] = None):
    """dict(drows [..., width], dwq, dwk), and for each `mag_*`: the sum of the magnitudes of the
    terms that make an element, which a rounding error of its float32 sum is relative to."""
    q, k, _, _ = split(p, rows)
    parts, mags, out = [], [], {}
    for x, w, up, name in ((q, wq, dq, "q"), (k, wk, dk, "k")):
        size = np.abs(up)
        if name == "k":
            up, size = _shared(p, up), _shared(p, size)
        g = turn(up, cs, back=True)
        pair = np.repeat(size[..., 0::2] + size[..., 1::2], 2, axis=-1) if cs is not None else size
        y, r = rms(p, x)
        if w is not None:
            out["dw" + name] = (g * y).sum((0, 1, 2, 3, 4))
            out["mag_dw" + name] = (pair * np.abs(y)).sum((0, 1, 2, 3, 4))
            g, pair = g * w, pair * np.abs(w)
        if p.norm:
            mags.append(_rows_of(r * (pair + np.abs(y) * np.mean(pair * np.abs(y), axis=-1, keepdims=True))))
            g = r * (g - y * np.mean(g * y, axis=-1, keepdims=True))
        else:
            mags.append(_rows_of(pair))
        parts.append(_rows_of(g))
    parts.append(_rows_of(_shared(p, dv)))
    mags.append(_rows_of(_shared(p, np.abs(dv))))
    if dgate is not None:
        g = np.moveaxis(dgate, 1, 4) if p.gate == 1 else _rows_of(dgate)
        parts.append(g)
        mags.append(np.abs(g))
    out["drows"] = np.concatenate(parts, axis=-1)
    out["mag_drows"] = np.concatenate(mags, axis=-1)
    return out
