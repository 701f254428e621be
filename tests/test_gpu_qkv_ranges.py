"""The rows' backward at the ends of its ranges."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2606_31248_amd import binding as B

from _rows import ARITH, HALF_STEP, Case, Problem, TYPE, f64, gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_heads_without_eps(dtype, codes):
    """eps = 0 and heads of 2^-66, among ordinary ones: the reciprocal root is 2^66, its square beyond float32.  Their
    squares are subnormal, each off by up to 2^-150: 2^-149 of a mean of 2^-133 and more, so 2^-17 of the reciprocal
    root, three times in a gradient: below 2^-15 of its terms."""
    c = Case(dtype, 1, 4, 2, 1, 2, 4, 64, gate=64)
    x = Problem(c, 31)
    x.desc.eps = 0.0
    x.rows = normal(tuple(x.rows.shape), dtype, gen(32))
    x.rows *= torch.tensor([2.0 ** -66, 1.0, 2.0 ** -64, 2.0 ** -66] * 2).view(1, 1, 2, 4, 1).to(TYPE[dtype]).cuda()
    kept = x.codes_out() if codes else (None, None)
    out = x.forward(*kept)
    got = x.backward(None if codes else x.rows, *kept)
    x.check_guards()
    if codes:
        held = torch.empty(c.grid + (c.p.kept,), dtype=TYPE[dtype], device="cuda")
        B.strata_ckpt_unpack(*kept, held)
        again, x.rows = x.again(*kept), held.contiguous()
        out = dict(out, q=again["q"], k=again["k"])
    p = dataclasses.replace(c.p, eps=0.0)
    q, k = R.split(p, x.rows64())[:2]
    assert min(np.mean(y * y, axis=-1).min() for y in (q, k)) > 2.0 ** -133
    want = R.forward(p, x.rows64(), f64(x.wq), f64(x.wk), f64(x.cs))
    for n in ("q", "k"):
        pair = np.repeat(np.abs(want[n][..., 0::2]) + np.abs(want[n][..., 1::2]), 2, axis=-1)
        assert np.all(np.abs(f64(out[n]) - want[n]) <= HALF_STEP[dtype] * np.abs(want[n]) + 2.0 ** -15 * pair), n
    want = R.backward(p, x.rows64(), wq=f64(x.wq), wk=f64(x.wk), cs=f64(x.cs), **{n: f64(t) for n, t in x.up.items()})
    tol = HALF_STEP[dtype] * np.abs(want["drows"]) + (2.0 ** -15 + 2 * ARITH) * want["mag_drows"]
    assert np.all(np.abs(f64(got["drows"])[..., :c.p.width] - want["drows"]) <= tol)
    for n in ("dwq", "dwk"):
        assert np.all(np.abs(f64(got[n]) - want[n]) <= 2.0 ** -15 * want["mag_" + n])
