"""Oracle: the residual stream's norm with its gradients, the norm of gradients, AdamW and
its states in 8 bits (test infrastructure, CPU only, numpy float64).

Rows are [groups, group_rows, width], vectors [groups, width].
"""
from __future__ import annotations

import numpy as np


# ---- residual addition and RMS norm ------------------------------------------------

def add(res, x=None, gate=None):
    if x is None:
        return res
    return res + (x if gate is None else gate[:, None] * x)


def norm(total, scale=None, shift=None, eps=1e-6):
    """(y, the normalised rows, 1 / root mean square) of the stored sum."""
    r = 1.0 / np.sqrt(np.mean(total * total, axis=-1, keepdims=True) + eps)
    n = total * r
    y = n if scale is None else n * scale[:, None]
    return (y if shift is None else y + shift[:, None]), n, r


def norm_backward(total, dy, dsum=None, x=None, gate=None, scale=None, eps=1e-6):
    """dict(dres, dx, dgate, dscale, dshift), and for each `mag_*`: the sum of the magnitudes of the terms that make
    an element, which the rounding errors of its float32 arithmetic are relative to."""
    _, n, r = norm(total, eps=eps)
    w = 1.0 if scale is None else scale[:, None]
    u = r * w * dy
    h = u - n * np.mean(u * n, axis=-1, keepdims=True)
    mag = np.abs(u) + np.abs(n) * np.mean(np.abs(u * n), axis=-1, keepdims=True)
    if dsum is not None:
        h, mag = h + dsum, mag + np.abs(dsum)
    out = dict(dres=h, mag_dres=mag, dscale=(dy * n).sum(1), mag_dscale=np.abs(dy * n).sum(1), dshift=dy.sum(1),
               mag_dshift=np.abs(dy).sum(1))
    if gate is not None:
        out.update(dx=h * gate[:, None], mag_dx=mag * np.abs(gate[:, None]), dgate=(h * x).sum(1),
                   mag_dgate=(mag * np.abs(x)).sum(1))
    return out


# ---- AdamW ---------------------------------------------------------------------------

def adamw(p, g, m, v, lr, step, beta1, beta2, eps, decay):
    """(p, m, v) after the step."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p - lr * (decay * p + (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)), m, v


def moments32(g, m, v, beta1, beta2):
    """m and v in float32, every product and sum rounded by itself."""
    f = np.float32
    g, m, v = f(g), f(m), f(v)
    with np.errstate(over="ignore", invalid="ignore"):
        return f(beta1) * m + f(1 - beta1) * g, f(beta2) * v + f(1 - beta2) * g * g


UNIT = {False: 17, True: 33}   # octaves from the exponent of a group's largest to its unit; True: the second moment


def encode(x, random, second):
    """float32 values in whole groups of 32 and numbers in [0, 1) -> (codes, exponents)."""
    v = np.asarray(x, np.float32).reshape(-1, 32)
    fine = np.isfinite(v).all(1)
    a = np.where(fine[:, None], np.abs(v), 0).astype(np.float64)
    top = a.max(1)
    e = np.where(top > 0, np.frexp(top)[1] + 126, 0)                   # top = f 2^(e - 126), 1/2 <= f < 1
    e = np.where(np.ldexp(top, 126 - e) >= 15 / 16, e + 1, e)
    e = np.clip(e, UNIT[second] + 1, 254)
    t = np.ldexp(a, (127 + UNIT[second] - e)[:, None])                 # in units, exact
    octave = np.maximum(np.frexp(t)[1] - 1, 3)
    # in steps: the sum below 8 is rounded as float32 rounds it, above it is exact
    part = np.floor((np.ldexp(t, 3 - octave).astype(np.float32) + np.asarray(random, np.float32).reshape(-1, 32)))
    code = (octave - 3) * 8 + part.astype(np.int64)
    code = np.minimum(code, 255 if second else 127)                    # at the largest exponent
    if second:
        code = np.where(a > 0, np.maximum(code, 1), code)
    else:
        code = code + np.where(np.signbit(v), 128, 0)
    code = np.where(fine[:, None], code, 0)
    return code.astype(np.uint8).reshape(-1), np.where(fine, e, 255).astype(np.uint8)


def decode(codes, scales, second):
    """Float64 values of codes (the last group may be short)."""
    c = np.asarray(codes, np.int64)
    s = np.repeat(np.asarray(scales, np.int64), 32)[:c.size]
    k = c if second else c & 127
    f = np.where(k < 8, k, (8 + (k & 7)) * 2.0 ** ((k >> 3) - 1.0))
    v = f * 2.0 ** (np.maximum(s - UNIT[second], 1) - 127.0)
    if not second:
        v = np.where(c >= 128, -v, v)
    return np.where(s == 255, np.nan, v)


def _mix(x):
    m = 0xFFFFFFFF
    x = (x ^ x >> 16) * 0x6A09E667 & m
    x = (x ^ x >> 15) * 0xBB67AE85 & m
    return x ^ x >> 16


def random_numbers(seed, places):
    """The two numbers in [0, 1) of each place: for m and for v."""
    key = _mix(_mix((seed & 0xFFFFFFFF) + 0x3C6EF372 & 0xFFFFFFFF) ^ seed >> 32)
    x = np.asarray(places, np.uint64) ^ np.uint64(key)
    m = np.uint64(0xFFFFFFFF)
    for factor, shift in ((0x6A09E667, 16), (0xBB67AE85, 15)):
        x = (x ^ x >> np.uint64(shift)) * np.uint64(factor) & m
    x = x ^ x >> np.uint64(16)
    return (x & np.uint64(0xFFFF)).astype(np.float32) / 65536, (x >> np.uint64(16)).astype(np.float32) / 65536
