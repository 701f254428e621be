"""Projection rows into the head layout and back (strata_qkv_heads, _ckpt, _bwd)
against the float64 oracle: types, head layouts, odd grids, one token, padding."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_2606_31248_amd import binding as B

from _rows import Case, Problem, TYPE, check_grads, check_heads, gen, normal, phases

pytestmark = pytest.mark.gpu

CASES = [
    Case("bf16", 1, 1, 1, 1, 1, 1, 64),                                   # one token, one head
    Case("f32", 1, 3, 1, 1, 1, 1, 32, gate=1),
    Case("bf16", 1, 16, 16, 1, 1, 1, 128, gate=128, pad=8),
    Case("bf16", 2, 4, 4, 3, 5, 7, 64),                                   # 105 tokens: a wave's 8 straddle the tiles
    Case("bf16", 3, 4, 2, 1, 3, 3, 64, gate=1, pad=24),
    Case("bf16", 2, 11, 11, 2, 3, 5, 64, gate=64),
    Case("bf16", 5, 6, 1, 1, 1, 3, 32, gate=32, pad=40),                  # fewer tokens a tile than a wave takes
    Case("bf16", 1, 2, 2, 3, 9, 5, 128, gate=1, norm=False, weights=False),
    Case("f32", 2, 4, 2, 3, 5, 7, 64, gate=64, pad=4),
    Case("f32", 1, 8, 8, 2, 3, 3, 128, rope=False),
    Case("f32", 1, 16, 4, 2, 5, 5, 32, gate=1, weights=False),
    Case("bf16", 1, 4, 4, 2, 5, 5, 64, rope=False, norm=False, weights=False),   # layout alone
    Case("bf16", 2, 16, 16, 4, 16, 16, 64, gate=64),                      # many waves
    Case("bf16", 1, 3, 3, 24, 33, 31, 32, gate=1),
    # rows off the cache lines with heads enough to lie beside each other in a wave of the backward
    Case("bf16", 2, 16, 16, 2, 5, 7, 64, gate=64, pad=8),
    Case("bf16", 1, 11, 11, 3, 5, 5, 64, gate=64, pad=16),                # 11 of 12 places taken
    Case("bf16", 2, 16, 4, 3, 5, 3, 64, gate=1),
    Case("bf16", 1, 16, 8, 2, 5, 9, 32, gate=32, pad=8),
    Case("bf16", 3, 4, 2, 1, 7, 3, 128, gate=1, weights=False),
    Case("bf16", 1, 4, 4, 2, 5, 3, 128, gate=128, pad=8),
    Case("bf16", 1, 16, 16, 1, 5, 3, 32, gate=32, pad=16),
    Case("bf16", 2, 6, 6, 1, 3, 5, 64, gate=64, pad=8),
    Case("bf16", 1, 2, 2, 3, 3, 3, 64, gate=1),
    Case("f32", 1, 8, 4, 2, 5, 3, 64, gate=1),
    # shared heads in several rounds of loads
    Case("bf16", 1, 10, 2, 2, 3, 5, 64),
    Case("bf16", 2, 16, 1, 1, 4, 9, 64, gate=1),
    Case("f32", 1, 7, 1, 2, 3, 5, 32, gate=32),
    Case("bf16", 1, 70, 35, 1, 2, 3, 32, gate=1),                         # more logits a token than lanes
]
IDS = [f"{c.dtype}-{c.B}x{c.heads}.{c.kv}x{c.Z}x{c.H}x{c.W}x{c.d}-g{c.gate}p{c.pad}" for c in CASES]


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_forward(c):
    x = Problem(c)
    out = x.forward()
    x.check_guards()
    check_heads(out, x.want_forward(x.rows64()), c.dtype, "forward")


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_forward_with_eight_bits_and_again(c):
    """The 8-bit form beside the forward, which it does not change; the heads made again from it equal the
    forward of the rows that it stands for, bit for bit."""
    x = Problem(c, 1)
    plain = x.forward()
    codes, scales = x.codes_out()
    out = x.forward(codes, scales)
    again = x.again(codes, scales)
    x.check_guards()
    for n in plain:
        assert plain[n] is None or torch.equal(plain[n], out[n])
    want = R.encode(x.rows64()[..., :c.p.kept])
    assert np.array_equal(codes.cpu().numpy().reshape(-1), want[0])
    assert np.array_equal(scales.cpu().numpy().reshape(-1), want[1])
    held = torch.from_numpy(R.decode(*want)).view(c.grid + (c.p.kept,))
    x.rows[..., :c.p.kept] = held.to(TYPE[c.dtype]).cuda()
    assert np.array_equal(x.rows64()[..., :c.p.kept], held.numpy())       # exact in both types
    other = x.forward()
    for n in ("q", "k", "v") + (("gate",) if c.gate > 1 else ()):
        assert torch.equal(again[n], other[n]), n


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_backward(c):
    x = Problem(c, 2)
    got = x.backward(x.rows)
    x.check_guards()
    check_grads(got, x.want_backward(x.rows64()), c.dtype, "backward")
    assert bool((got["drows"][..., c.p.width:] == 7).all()), "padding written"


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_backward_from_eight_bits(c):
    """The gradient at the values the codes stand for, whatever the rows were; equal bit for bit to the
    backward from rows that hold them."""
    x = Problem(c, 3)
    codes, scales = x.codes_out()
    x.forward(codes, scales)
    got = x.backward(None, codes, scales)
    held = R.decode(*R.encode(x.rows64()[..., :c.p.kept])).reshape(c.grid + (c.p.kept,))
    rows64 = np.concatenate([held, x.rows64()[..., c.p.kept:]], -1)
    x.rows[..., :c.p.kept] = torch.from_numpy(held).to(TYPE[c.dtype]).cuda()
    other = x.backward(x.rows)
    x.check_guards()
    check_grads(got, x.want_backward(rows64), c.dtype, "backward from 8 bits")
    assert torch.equal(got["drows"][..., :c.p.width], other["drows"][..., :c.p.width])
    for n in ("dwq", "dwk"):
        assert got[n] is None or torch.equal(got[n], other[n])


def test_backward_of_many_tokens_with_one_head():
    """70656 tokens of one 128-channel head: a wave takes several tiles, the weights' sums two launches."""
    c = Case("bf16", 1, 1, 1, 24, 64, 46, 128, gate=0)
    x = Problem(c, 11)
    got = x.backward(x.rows)
    x.check_guards()
    want = x.want_backward(x.rows64())
    # here the sums have up to 5 additions in a lane, 2 in a block and 50 in the two sums: within WEIGHT_SUM
    check_grads(got, want, c.dtype, "backward")


@pytest.mark.parametrize("codes", [False, True])
def test_many_tiles_equal_each_tile_alone(codes):
    """Rows past 2^29 elements (and offsets past 2^32 bytes): the same bits as tile by tile."""
    c = Case("bf16", 9, 16, 16, 8, 64, 64, 64, gate=64)
    g = torch.Generator(device="cuda").manual_seed(12)
    rows = torch.empty(c.grid + (4096,), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    cs = phases(c, gen(13))
    w = torch.linspace(0.5, 1.5, 64, device="cuda")

    def run(b, r, table):
        one = dataclasses.replace(c, B=b)
        out = [torch.empty(one.shape, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
        kept = [torch.empty(one.grid + (4096,), dtype=torch.int8, device="cuda"),
                torch.empty(one.grid + (128,), dtype=torch.uint8, device="cuda")] if codes else [None, None]
        B.strata_qkv_heads(one.desc(), r, w, w, table, *out, *kept)
        return out + [t for t in kept if t is not None]

    whole = run(9, rows, cs)
    for b in (0, 4, 8):
        for got, want in zip(whole, run(1, rows[b:b + 1].contiguous(), cs[b:b + 1].contiguous())):
            assert torch.equal(got[b:b + 1], want)


def test_gradient_against_differences():
    """<dout, f(x + h e) - f(x - h e)> of the kernels' own float32 forward.  A difference over 2h with
    h = 2^-6 has a truncation error of h^2/6 of a third derivative (order one for rows of unit size:
    below 2^-13) and a rounding error of about 2^-24 sqrt(n) |dout| |f| / h, n = 3 heads of 32: below 2^-14."""
    c = Case("f32", 1, 1, 1, 1, 1, 1, 32)
    x = Problem(c, 4)
    x.rows = normal(c.grid + (x.desc.row_stride,), "f32", gen(9))
    got = x.backward(x.rows)
    base, h = x.rows.clone(), 2.0 ** -6
    for i in range(0, c.p.width, 5):
        vals = []
        for sign in (1, -1):
            x.rows = base.clone()
            x.rows[..., i] += sign * h
            o = x.forward()
            vals.append(sum(float((o[n].double() * x.up["d" + n].double()).sum()) for n in ("q", "k", "v")))
        diff = (vals[0] - vals[1]) / (2 * h)
        assert abs(diff - float(got["drows"].reshape(-1)[i])) < 2.0 ** -10


def test_repeated_calls_agree_bit_for_bit():
    x = Problem(CASES[12], 5)
    a, b = x.backward(x.rows), x.backward(x.rows)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_rows(dtype):
    """Zero heads, tiny heads and large heads: eps decides, nothing overflows below 2^60."""
    c = Case(dtype, 1, 4, 2, 1, 2, 4, 64)
    x = Problem(c, 6)
    size = torch.tensor([0.0, 2.0 ** -40, 2.0 ** 40, 1.0, 2.0 ** -10, 1.0, 0.0, 2.0 ** 20]).view(1, 1, 2, 4, 1)
    x.rows *= size.to(TYPE[dtype]).cuda()
    out, got = x.forward(), x.backward(x.rows)
    check_heads(out, x.want_forward(x.rows64()), dtype, "forward")
    check_grads(got, x.want_backward(x.rows64()), dtype, "backward")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_rows_in_eight_bits(dtype):
    """Heads from 0 to the largest finite values, whose squares overflow or vanish, in 8 bits: heads made again and
    gradients equal those of rows that hold the decoded values (with NaN where they have NaN)."""
    c = Case(dtype, 1, 4, 2, 1, 2, 6, 64, gate=64)
    x = Problem(c, 14)
    x.rows = normal(tuple(x.rows.shape), dtype, gen(15)).clamp(-1.5, 1.5)
    size = torch.tensor([0.0, 2.0 ** -126, 2.0 ** -100, 2.0 ** -63, 2.0 ** -20, 1.0, 2.0 ** 20, 2.0 ** 62, 2.0 ** 64, 2.0 ** 100,
                         2.0 ** 125, 2.0 ** 127]).view(1, 1, 2, 6, 1)
    x.rows *= size.to(TYPE[dtype]).cuda()
    codes, scales = x.codes_out()
    x.forward(codes, scales)
    assert int(scales.max()) == 254 and int(scales.min()) == 7
    again, got = x.again(codes, scales), x.backward(None, codes, scales)
    held = torch.empty(c.grid + (c.p.kept,), dtype=TYPE[dtype], device="cuda")
    B.strata_ckpt_unpack(codes, scales, held)
    x.rows = held.contiguous()
    other, want = x.forward(), x.backward(x.rows)
    same = lambda a, b: bool(((a == b) | (a.isnan() & b.isnan())).all())  # noqa: E731
    for n in other:
        assert same(again[n], other[n]), n
    for n in want:
        assert same(got[n], want[n]), n


def test_zero_heads_without_eps():
    """eps = 0: a zero head has no norm (NaN), from rows and from 8 bits, and its neighbours keep theirs."""
    c = Case("bf16", 1, 4, 4, 1, 2, 4, 64)
    x = Problem(c, 16)
    x.desc.eps = 0.0
    x.rows[0, 0, 1, 2, 64:128] = 0
    codes, scales = x.codes_out()
    out, again = x.forward(codes, scales), x.again(codes, scales)
    for o in (out, again):
        bad = o["q"].isnan().any(-1)
        assert int(bad.sum()) == 1 and bool(bad[0, 1, 0, 1, 2]) and not o["k"].isnan().any()


def test_a_broken_row_stays_alone():
    """A NaN or an infinity in one head reaches that head of that token and, in 8 bits, its group of 32."""
    c = Case("bf16", 1, 4, 2, 1, 4, 8, 64, gate=64)
    x = Problem(c, 7)
    x.rows[0, 0, 1, 2, 64 + 3] = float("nan")        # query head 1 of token (1, 2)
    x.rows[0, 0, 3, 5, 4 * 64 + 40] = float("inf")   # key head 0 of token (3, 5)
    codes, scales = x.codes_out()
    out = x.forward(codes, scales)
    bad_q, bad_k = torch.isnan(out["q"]).any(-1), ~torch.isfinite(out["k"]).all(-1)
    assert bad_q.sum() == 1 and bool(bad_q[0, 1, 0, 1, 2])
    assert bad_k.sum() == 2 and bool(bad_k[0, :2, 0, 3, 5].all())
    assert (scales == 255).sum() == 2
    assert int(scales[0, 0, 1, 2, 2]) == 255 and int(scales[0, 0, 3, 5, (4 * 64 + 40) // 32]) == 255
    again = x.again(codes, scales)
    assert torch.equal(torch.isnan(again["q"]).any(-1), bad_q)
    assert torch.equal(torch.isnan(again["k"]).any(-1), bad_k)


def test_another_stream():
    x = Problem(CASES[12], 8)
    want = {n: t.clone() for n, t in x.forward().items()}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o = x.heads_out()
    torch.cuda.synchronize()
    B.strata_qkv_heads(x.desc, x.rows, x.wq, x.wk, x.cs, o["q"], o["k"], o["v"], o["gate"], stream=s)
    s.synchronize()
    for n in want:
        assert torch.equal(want[n], o[n]), n


def test_captured_and_replayed():
    """Forward with 8 bits and the backward from them in one graph, with eager calls between the replays."""
    x = Problem(CASES[12], 9)
    codes, scales = x.codes_out()
    o, t = x.heads_out(), TYPE["bf16"]
    drows = torch.zeros_like(x.rows)
    dwq, dwk = torch.zeros_like(x.wq), torch.zeros_like(x.wk)
    ws = torch.empty(B.strata_qkv_heads_bwd_workspace_size(x.desc), dtype=torch.uint8, device="cuda")

    def step():
        B.strata_qkv_heads(x.desc, x.rows, x.wq, x.wk, x.cs, o["q"], o["k"], o["v"], o["gate"], codes, scales)
        B.strata_qkv_heads_bwd(x.desc, None, codes, scales, x.wq, x.wk, x.cs, x.up["dq"], x.up["dk"], x.up["dv"],
                               x.up["dgate"], drows, dwq, dwk, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (20, 21, 22):
        x.rows.copy_(normal(tuple(x.rows.shape), "bf16", gen(seed)))
        eager_codes = torch.empty_like(codes), torch.empty_like(scales)
        want = x.forward(*eager_codes)
        grads = x.backward(None, *eager_codes)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(want[n], o[n]), n
        assert torch.equal(codes, eager_codes[0]) and torch.equal(scales, eager_codes[1])
        assert torch.equal(grads["drows"][..., :x.c.p.width], drows[..., :x.c.p.width])
        assert torch.equal(grads["dwq"], dwq) and torch.equal(grads["dwk"], dwk)


def test_binding_refusals():
    x = Problem(CASES[4], 10)
    d, o = x.desc, x.heads_out()
    codes, scales = x.codes_out()
    call = lambda **kw: B.strata_qkv_heads(**{**dict(desc=d, rows=x.rows, wq=x.wq, wk=x.wk, cs=x.cs, **o), **kw})  # noqa: E731
    half = lambda t: t[..., :t.shape[-1] // 2].contiguous()  # noqa: E731
    for kw in (dict(rows=half(x.rows)), dict(rows=x.rows.float()), dict(q=half(o["q"])), dict(k=o["k"].float()),
               dict(v=o["v"].cpu()), dict(gate=o["q"]), dict(cs=half(x.cs)), dict(wq=x.wq.bfloat16()),
               dict(wk=x.wk[:32].contiguous()), dict(rows=x.rows.transpose(2, 3).contiguous().transpose(2, 3)),
               dict(codes=half(codes), scales=scales), dict(codes=codes, scales=codes)):
        with pytest.raises(ValueError):
            call(**kw)
    call(rows=x.rows.transpose(1, 2).contiguous().transpose(1, 2))  # an axis of one element: the same memory
    with pytest.raises(B.StrataError):
        call(gate=None)
    with pytest.raises(B.StrataError):
        call(codes=codes)
    with pytest.raises(B.StrataError):  # a workspace one byte short
        B.strata_qkv_heads_bwd(d, x.rows, None, None, x.wq, x.wk, x.cs, x.up["dq"], x.up["dk"], x.up["dv"],
                               x.up["dgate"], torch.empty_like(x.rows), torch.empty_like(x.wq), torch.empty_like(x.wk),
                               torch.empty(15, dtype=torch.uint8, device="cuda"))
