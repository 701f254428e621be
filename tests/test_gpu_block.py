"""One attention block from its projection's rows to their gradient (pipeline.block_forward,
block_backward): against the oracle's chain, and from 8 bits against the same chain at the
values that the codes stand for."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rows as R
from paper_2606_31248_amd import binding as B
from paper_2606_31248_amd import pipeline

from _rows import ARITH, HALF_STEP, Case, Problem, f64, gen, normal
from _util import BF16_REL_RMS, F32_ABS, bf16_half_ulp, check_close

pytestmark = pytest.mark.gpu

CASES = [
    (Case("bf16", 2, 4, 2, 8, 12, 10, 64, gate=64), (3, 7, 7)),
    (Case("bf16", 1, 3, 3, 9, 9, 11, 64, gate=1, pad=8), (9, 9, 9)),
    (Case("bf16", 1, 2, 1, 6, 5, 5, 64, rope=False), (6, 1, 1)),
    (Case("f32", 1, 2, 1, 3, 7, 9, 32, gate=1), (3, 5, 7)),
]


def attention64(c, window, o, dout=None, want_lse=False):
    """The oracle's attention on head-layout values (plain: norm and rotation are done), gate included."""
    gate = o.get("gate")
    out, lse = oracle.na3d_fwd(o["q"], o["k"], o["v"], window, c.d ** -0.5, gate=gate)
    if dout is None:
        return out, lse
    return oracle.na3d_bwd(o["q"], o["k"], o["v"], dout, window, c.d ** -0.5, gate=gate)


@pytest.mark.parametrize("c,window", CASES)
def test_block_against_the_oracle(c, window):
    """Rows kept as they are.  The oracle's chain takes the q, k, v and gate that strata_qkv_heads made (held to one
    rounding of the exact ones elsewhere): a rounding of q and k moves a logit of a peaked row, and with it an output
    near 1 by several 2^-9, which is no error of the attention."""
    x = Problem(c, 1)
    x.rows = normal(tuple(x.rows.shape), c.dtype, gen(31))
    out, saved = pipeline.block_forward(x.rows, x.desc, window, c.d ** -0.5, x.wq, x.wk, x.cs)
    dout = normal(c.shape, c.dtype, gen(30))
    drows, dwq, dwk = pipeline.block_backward(saved, dout)
    rows64 = x.rows64()
    heads = {n: f64(t) for n, t in x.forward().items() if t is not None}
    want, _ = attention64(c, window, heads)
    check_close(f64(out), want, c.dtype, "out")
    grads = attention64(c, window, heads, f64(dout))
    names = ("dq", "dk", "dv", "dgate")
    up = dict(zip(names, grads))
    want = R.backward(c.p, rows64, wq=f64(x.wq), wk=f64(x.wk), cs=f64(x.cs), **up)
    # the library's rule for each head-layout gradient, its own rounding included, carried through the rows'
    # backward: |J| times it, which mag_drows is for the magnitudes given; then that backward's own rounding
    rule = {n: F32_ABS * np.ones_like(g) if c.dtype == "f32" else BF16_REL_RMS * np.sqrt(np.mean(g * g)) + bf16_half_ulp(g)
            for n, g in up.items()}
    rule.setdefault("dgate", None)
    tol = R.backward(c.p, rows64, wq=f64(x.wq), wk=f64(x.wk), cs=f64(x.cs), **rule)["mag_drows"]
    tol += HALF_STEP[c.dtype] * np.abs(want["drows"]) + 2 * ARITH * want["mag_drows"]
    worst = np.max(np.abs(f64(drows)[..., :c.p.width] - want["drows"]) - tol)
    assert worst <= 0, f"drows off by {worst:.3e} more than its tolerance"
    assert bool((drows[..., c.p.width:] == 0).all())
    for got, ref in ((dwq, want["dwq"]), (dwk, want["dwk"])):
        err = np.linalg.norm(f64(got) - ref) / np.linalg.norm(ref)
        assert err <= (4e-5 if c.dtype == "f32" else 2e-2), err


@pytest.mark.parametrize("c,window", CASES)
def test_block_from_eight_bits(c, window):
    """The same forward bit for bit; the backward equals the chain on rows and output that hold the decoded values."""
    x = Problem(c, 2)
    run = lambda eight: pipeline.block_forward(x.rows, x.desc, window, c.d ** -0.5, x.wq, x.wk, x.cs, eight_bit=eight)  # noqa: E731
    out, plain = run(False)
    out8, saved = run(True)
    assert torch.equal(out, out8) and torch.equal(plain.lse, saved.lse)
    dout = normal(c.shape, c.dtype, gen(40))
    got = pipeline.block_backward(saved, dout)
    held = x.rows.clone()
    kept = torch.empty(c.grid + (c.p.kept,), dtype=held.dtype, device="cuda")
    B.strata_ckpt_unpack(*saved.rows, kept)
    held[..., :c.p.kept] = kept
    out_held = torch.empty_like(out)
    B.strata_ckpt_unpack(*saved.out, out_held)
    plain.rows, plain.out = held, out_held
    want = pipeline.block_backward(plain, dout)
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    # 8 bits and a scale for 32 of them against 16 (or 32), the lse and one-per-head gate logits as they are
    e = x.rows.element_size()
    full = c.B * c.Z * c.H * c.W * (x.desc.row_stride + c.heads * c.d) * e
    other = saved.lse.numel() * 4 + (saved.gate.numel() * e if saved.gate is not None else 0)
    assert saved.nbytes() - other <= full * (33 / 32) / e + 32


def test_eight_bit_gradient_is_close():
    """How far 8 bits move a gradient.  Rows are off by 0.9 % of their size (a step of at most A/64, A about 2.1 of
    32 normal values, over sqrt(12)), twice in a logit of unit deviation (q and k: 1.3 %), and as much again in v, out
    and the norm's own backward: four such independent parts stay under 4 %."""
    c, window = CASES[0]
    x = Problem(c, 3)
    x.rows = normal(tuple(x.rows.shape), c.dtype, gen(50))
    dout = normal(c.shape, c.dtype, gen(51))
    grads = []
    for eight in (False, True):
        _, saved = pipeline.block_forward(x.rows, x.desc, window, c.d ** -0.5, x.wq, x.wk, x.cs, eight_bit=eight)
        grads.append(pipeline.block_backward(saved, dout)[0].double())
    assert float((grads[1] - grads[0]).norm() / grads[0].norm()) < 0.04


def test_block_replays():
    """Forward and backward from 8 bits captured into one graph, replayed on other rows between eager blocks."""
    c, window = CASES[0]
    x = Problem(c, 4)
    dout = normal(c.shape, c.dtype, gen(60))

    def block():
        out, saved = pipeline.block_forward(x.rows, x.desc, window, c.d ** -0.5, x.wq, x.wk, x.cs, eight_bit=True)
        return (out,) + pipeline.block_backward(saved, dout)

    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block()
    for seed in (61, 62, 63):
        x.rows.copy_(normal(tuple(x.rows.shape), c.dtype, gen(seed)))
        want = block()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w)
