"""The rows' backward at the ends of its ranges: heads whose squares leave float32's, more tokens than the card has
waves, rows past 2^32 bytes."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2606_31248_amd import binding as B

from _rows import ARITH, HALF_STEP, WEIGHT_SUM, Case, Problem, TYPE, check_grads, f64, gen, normal, phases

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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_whose_squares_overflow(dtype):
    """Heads of 2^64: a norm of 0 and a gradient of 0, no NaN, the other tokens as ever."""
    c = Case(dtype, 1, 4, 2, 1, 2, 4, 64)
    x = Problem(c, 33)
    x.rows = normal(tuple(x.rows.shape), dtype, gen(34))
    plain, other = x.forward(), x.backward(x.rows)
    x.rows[0, 0, 1, 2, :8 * 64] *= 2.0 ** 64
    out, got = x.forward(), x.backward(x.rows)
    for n in ("q", "k"):
        assert not out[n][0, :, 0, 1, 2].any()
        plain[n][0, :, 0, 1, 2] = 0
        assert torch.equal(out[n], plain[n])
    assert not got["drows"][0, 0, 1, 2, :6 * 64].any()
    other["drows"][0, 0, 1, 2, :6 * 64] = 0
    assert torch.equal(got["drows"], other["drows"])
    assert got["dwq"].isfinite().all() and got["dwk"].isfinite().all()


# More waves than two rounds of the card's: a wave of the backward takes two or four tiles of tokens.
LONG = [
    (Case("bf16", 1, 1, 1, 24, 64, 43, 128, gate=128), True),            # from codes, one head
    (Case("f32", 1, 1, 1, 24, 64, 43, 128, gate=1), False),              # gate logits beside the norm's heads
    (Case("bf16", 1, 2, 2, 24, 64, 43, 64, gate=1), False),              # two heads beside each other off the lines
    (Case("bf16", 1, 2, 2, 24, 64, 43, 64, gate=1), True),
    (Case("bf16", 2, 4, 2, 8, 45, 47, 128), False),                      # shared heads
    (Case("bf16", 2, 4, 2, 8, 45, 47, 128, gate=1), True),               # shared, beside each other, from codes
]


@pytest.mark.parametrize("c,codes", LONG)
def test_backward_with_several_tiles_a_wave(c, codes):
    """Against the oracle, and drows bit for bit as level by level, in calls too small for a second tile."""
    x = Problem(c, 35)
    kept = x.codes_out() if codes else (None, None)
    if codes:
        x.forward(*kept)
        held = R.decode(kept[0].cpu().numpy().reshape(-1), kept[1].cpu().numpy().reshape(-1))
        x.rows[..., :c.p.kept] = torch.from_numpy(held).view(c.grid + (c.p.kept,)).to(TYPE[c.dtype]).cuda()
    got = x.backward(None if codes else x.rows, *kept)
    x.check_guards()
    check_grads(got, x.want_backward(x.rows64()), c.dtype, "backward")
    for z in range(c.Z):                                                 # one level at a time
        one = Problem(dataclasses.replace(c, Z=1), 36)
        one.cs, one.wq, one.wk = x.cs, x.wq, x.wk
        one.rows = x.rows[:, z:z + 1].contiguous()
        one.up = {n: None if t is None else t[:, :, z:z + 1].contiguous() for n, t in x.up.items()}
        cut = [None if t is None else t[:, z:z + 1].contiguous() for t in kept]
        part = one.backward(None if codes else one.rows, *cut)["drows"]
        assert torch.equal(part[..., :c.p.width], got["drows"][:, z:z + 1, ..., :c.p.width]), z


@pytest.mark.parametrize("codes,pad", [(False, 0), (True, 0), (False, 8)])
def test_backward_past_32_bit_offsets(codes, pad):
    """Rows past 2^29 elements and 2^32 bytes would be 9 of these tiles': gradients as tile by tile, the weights'
    the sums in float64."""
    c = Case("bf16", 9, 16, 16, 8, 64, 64, 64, gate=64, pad=pad)
    g = torch.Generator(device="cuda").manual_seed(37)
    new = lambda shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    d = c.desc()
    rows, cs, w = new(c.grid + (d.row_stride,)), phases(c, gen(38)), torch.linspace(0.5, 1.5, 64, device="cuda")
    kept = [None, None]
    if codes:
        kept = [torch.empty(c.grid + (4096,), dtype=torch.int8, device="cuda"),
                torch.empty(c.grid + (128,), dtype=torch.uint8, device="cuda")]
        B.strata_ckpt_pack(rows, *kept)
        B.strata_ckpt_unpack(*kept, rows)
    ups = [new(c.shape) for _ in range(4)]

    def run(b, r, table, up, k):
        desc = dataclasses.replace(c, B=b).desc()
        out = [torch.full((b,) + c.grid[1:] + (desc.row_stride,), 7.0, dtype=torch.bfloat16, device="cuda"),
               torch.empty_like(w), torch.empty_like(w)]
        ws = torch.empty(B.strata_qkv_heads_bwd_workspace_size(desc), dtype=torch.uint8, device="cuda")
        B.strata_qkv_heads_bwd(desc, None if codes else r, *k, w, w, table, *up, *out, ws)
        return out

    whole = run(9, rows, cs, ups, kept)
    sums = np.zeros((4, 64))
    for b in range(9):
        at = lambda t: None if t is None else t[b:b + 1].contiguous()  # noqa: E731
        if b in (0, 4, 8):
            assert torch.equal(run(1, at(rows), at(cs), [at(t) for t in ups], [at(t) for t in kept])[0], whole[0][b:b + 1]), b
        co, si = (at(cs)[..., i].double()[:, None, None] for i in (0, 1))
        for i in range(2):
            up = ups[i][b:b + 1].double()
            x = rows[b:b + 1, ..., i * 1024:(i + 1) * 1024].unflatten(-1, (16, 64)).movedim(4, 1).double()
            y = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            e, o = up[..., 0::2], up[..., 1::2]
            back = torch.stack([e * co + o * si, o * co - e * si], -1).flatten(-2)
            pair = (e.abs() + o.abs()).repeat_interleave(2, -1)
            sums[i] += f64((back * y).sum((0, 1, 2, 3, 4)))
            sums[2 + i] += f64((pair * y.abs()).sum((0, 1, 2, 3, 4)))
    for i in range(2):
        assert np.all(np.abs(f64(whole[1 + i]) - sums[i]) <= WEIGHT_SUM * sums[2 + i])
    del whole, rows, ups, kept
    torch.cuda.empty_cache()
