"""Pins of the oracle's projection rows and 8-bit form: closed forms, and central
differences of its forward for its backward."""
import numpy as np
import pytest

from oracle import rows as R


def problem(p, seed=1, grid=(2, 2, 3, 2), rope=True):
    r = np.random.default_rng(seed)
    x = r.standard_normal(grid + (p.width,))
    th = r.uniform(-np.pi, np.pi, grid[:1] + grid[2:] + (p.d // 2,))
    cs = np.stack([np.cos(th), np.sin(th)], -1) if rope else None
    w = [1 + 0.3 * r.standard_normal(p.d) for _ in range(2)] if p.norm else [None, None]
    up = {n: r.standard_normal((grid[0], p.heads) + grid[1:] + (p.d,)) for n in ("dq", "dk", "dv")}
    up["dgate"] = r.standard_normal((grid[0], p.heads) + grid[1:] + ((p.d,) if p.gate > 1 else ())) if p.gate else None
    return x, cs, w, up


def test_forward_places_every_head():
    """Rows that hold their own index: the layout alone, with shared key heads."""
    p = R.Rows(heads=4, kv=2, d=4, gate=4, norm=False)
    grid = (2, 1, 2, 3)
    x = np.arange(np.prod(grid) * p.width, dtype=np.float64).reshape(grid + (p.width,))
    o = R.forward(p, x)
    for b in range(2):
        for h in range(4):
            for y in range(2):
                for c in range(3):
                    row = x[b, 0, y, c]
                    assert np.array_equal(o["q"][b, h, 0, y, c], row[4 * h:4 * h + 4])
                    assert np.array_equal(o["k"][b, h, 0, y, c], row[16 + 4 * (h // 2):20 + 4 * (h // 2)])
                    assert np.array_equal(o["v"][b, h, 0, y, c], row[24 + 4 * (h // 2):28 + 4 * (h // 2)])
                    assert np.array_equal(o["gate"][b, h, 0, y, c], row[32 + 4 * h:36 + 4 * h])


def test_norm_and_rotation_closed_forms():
    p = R.Rows(heads=1, kv=1, d=4, eps=0.0)
    x = np.tile(np.array([3.0, 4.0, -3.0, -4.0]), 3).reshape(1, 1, 1, 1, 12)
    quarter = np.zeros((1, 1, 1, 2, 2))
    quarter[..., 1] = 1.0  # (a, b) -> (-b, a)
    o = R.forward(p, x, cs=quarter)
    r = np.sqrt(12.5)      # mean square of 3, 4, 3, 4
    assert np.allclose(o["q"].reshape(-1), np.array([-4, 3, 4, -3]) / r, rtol=1e-15)
    assert np.array_equal(o["v"].reshape(-1), [3, 4, -3, -4])
    # eps under the root: rows of +-2 with eps = 5 are divided by 3
    y = np.full((1, 1, 1, 1, 12), 2.0)
    assert np.allclose(R.forward(R.Rows(1, 1, 4, eps=5.0), y)["k"], 2 / 3)


@pytest.mark.parametrize("p", [R.Rows(2, 2, 4), R.Rows(4, 2, 4, gate=1), R.Rows(3, 1, 4, gate=4, eps=0.1),
                               R.Rows(2, 1, 4, norm=False)])
def test_backward_against_central_differences(p):
    x, cs, (wq, wk), up = problem(p)
    got = R.backward(p, x, wq=wq, wk=wk, cs=cs, **up)

    def loss(x, wq, wk):
        o = R.forward(p, x, wq, wk, cs)
        return sum((o[n] * up["d" + n]).sum() for n in o)

    h = 1e-5
    r = np.random.default_rng(2)
    for _ in range(60):
        i = tuple(r.integers(0, n) for n in x.shape)
        e = np.zeros(x.shape)
        e[i] = h
        diff = (loss(x + e, wq, wk) - loss(x - e, wq, wk)) / (2 * h)
        assert abs(diff - got["drows"][i]) < 1e-7 * (1 + abs(diff))
    if p.norm:
        for n, w in (("dwq", 0), ("dwk", 1)):
            for c in range(p.d):
                e = np.zeros(p.d)
                e[c] = h
                a, b = ((wq + e, wk), (wq - e, wk)) if w == 0 else ((wq, wk + e), (wq, wk - e))
                diff = (loss(x, *a) - loss(x, *b)) / (2 * h)
                assert abs(diff - got[n][c]) < 1e-7 * (1 + abs(diff))
    for n in ("drows", "dwq", "dwk"):
        assert n not in got or np.all(got["mag_" + n] >= np.abs(got[n]) * (1 - 1e-12))


def test_eight_bits_closed_forms():
    x = np.zeros(96)
    x[0] = 127.0                # 127 steps of 1: the exponent of 1 is 127 + 6 = 133
    x[1], x[2], x[3] = 0.5, 1.5, -2.5
    x[32] = 127.5               # rounds to 128 steps of 1: steps of 2
    x[33], x[34] = 3.0, 63.0
    codes, scales = R.encode(x)
    assert list(scales) == [133, 134, 7]
    assert list(codes[:4]) == [127, 0, 2, -2]            # ties to even
    assert list(codes[32:35]) == [64, 2, 32]             # 63.75, 1.5, 31.5
    assert not codes[64:].any()
    v = R.decode(codes, scales)
    assert list(v[:4]) == [127.0, 0.0, 2.0, -2.0] and list(v[32:35]) == [128.0, 4.0, 64.0]


def test_eight_bits_error_and_extremes():
    r = np.random.default_rng(3)
    x = r.standard_normal(32 * 500) * 2.0 ** r.integers(-20, 20, 500).repeat(32)
    codes, scales = R.encode(x)
    err = np.abs(R.decode(codes, scales) - x)
    step = 2.0 ** (scales.astype(np.float64) - 133).repeat(32)
    assert np.all(err <= step / 2) and np.max(np.abs(codes)) <= 127
    assert np.all(np.abs(codes).reshape(-1, 32).max(1) >= 64)   # no bit of the step is wasted
    bad = np.array([1.0, np.inf, 2.0])
    assert R.encode(bad)[1][0] == 255 and not R.encode(bad)[0].any()
    assert np.isnan(R.decode(*R.encode(bad))).all()
    top = np.float64(np.finfo(np.float32).max)
    c, s = R.encode(np.array([top, -top, 1.0]))
    assert s[0] == 254 and list(c) == [127, -127, 0]
    c, s = R.encode(np.array([2.0 ** -126, 2.0 ** -127, 2.0 ** -149]))
    assert s[0] == 7 and list(c) == [1, 0, 0]
