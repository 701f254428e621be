"""Refusals of the residual norm, the weights' list and AdamW that need no GPU, and the table that a list makes;
the oracle's own rules for states in 8 bits."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import rows as R
from oracle import train as T
from paper_2606_31248_amd import binding as B

INVALID, UNSUPPORTED, WORKSPACE = B.STRATA_ERR_INVALID_ARG, B.STRATA_ERR_UNSUPPORTED, B.STRATA_ERR_WORKSPACE


def fake(addr=0x10000):
    return ctypes.c_void_p(addr)


def ref(d):
    return None if d is None else ctypes.byref(d)


# ---- residual norm -------------------------------------------------------------------

def desc(rows=96, group_rows=32, width=64, eps=1e-6, dtype=B.STRATA_BF16):
    return B.NormDesc(rows, group_rows, width, eps, dtype)


def fwd(d, x=fake(), gate=fake(), res=fake(), scale=fake(), shift=fake(), sum=fake(), y=fake(), codes=None, scales=None):
    return B.load().strata_residual_norm(ref(d), x, gate, res, scale, shift, sum, y, codes, scales, None)


def bwd(d, sum=fake(), x=fake(), gate=fake(), scale=fake(), dy=fake(), dsum=fake(), dres=fake(), dx=fake(), dgate=fake(),
        dscale=fake(), dshift=fake(), ws=fake(), nbytes=1 << 40):
    return B.load().strata_residual_norm_bwd(ref(d), sum, x, gate, scale, dy, dsum, dres, dx, dgate, dscale, dshift, ws,
                                             nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), INVALID), (dict(rows=-32), INVALID), (dict(rows=1 << 31, group_rows=1), INVALID),
    (dict(width=0), INVALID), (dict(width=-8), INVALID), (dict(width=8193), UNSUPPORTED), (dict(group_rows=0), INVALID),
    (dict(group_rows=-1), INVALID), (dict(group_rows=33), INVALID), (dict(group_rows=192), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(dtype=2), INVALID),
    (dict(rows=1 << 30, group_rows=1, width=1024), INVALID),           # 2^40 elements
])
def test_norm_descriptors(kw, status):
    d = desc(**kw)
    assert fwd(d) == status and B.load().strata_last_error() != b""
    assert bwd(d) == status
    assert B.strata_residual_norm_bwd_workspace_size(d) == 0


def test_norm_pointers():
    d = desc()
    assert fwd(None) == INVALID and bwd(None) == INVALID
    for kw in (dict(res=None), dict(sum=None), dict(x=None), dict(x=None, sum=None), dict(y=None), dict(codes=fake()),
               dict(scales=fake()), dict(codes=fake(0x10008), scales=fake()), dict(codes=fake(), scales=fake(0x10001)),
               dict(x=fake(0x10002)), dict(gate=fake(0x10004)), dict(scale=fake(0x10004)), dict(shift=fake(0x10008)),
               dict(sum=fake(0x10008)), dict(y=fake(0x10002)), dict(res=fake(0x10002))):
        assert fwd(d, **kw) == INVALID, kw
    assert fwd(desc(width=40), codes=fake(), scales=fake()) == INVALID          # groups of 32 would cross rows
    for kw in (dict(sum=None), dict(dy=None), dict(dres=None), dict(x=None), dict(dx=None), dict(dgate=None), dict(gate=None),
               dict(scale=None), dict(dscale=None), dict(sum=fake(0x10008)), dict(dy=fake(0x10008)), dict(dsum=fake(0x10002)),
               dict(dres=fake(0x10002)), dict(dx=fake(0x10002)), dict(dgate=fake(0x10004)), dict(dscale=fake(0x10004)),
               dict(dshift=fake(0x10004)), dict(ws=fake(0x10008))):
        assert bwd(d, **kw) == INVALID, kw


def test_norm_workspace():
    d = desc(rows=1 << 16, group_rows=1 << 16, width=512)
    need = B.strata_residual_norm_bwd_workspace_size(d)
    assert need > 0 and need % 256 == 0
    assert bwd(d, ws=None) == WORKSPACE and bwd(d, nbytes=255) == WORKSPACE
    # one row a group: its gradients are final
    assert B.strata_residual_norm_bwd_workspace_size(desc(group_rows=1)) == 0
    # partial sums stay under 16 MiB, or 10 % of what the rows move (five tensors)
    for rows, groups, width in ((1 << 18, 1, 1024), (1 << 12, 1, 8192), (8 * 98304, 8, 128), (15876, 4, 203), (64, 1, 8192),
                                (1 << 20, 1024, 128)):
        d = desc(rows=rows, group_rows=rows // groups, width=width)
        assert B.strata_residual_norm_bwd_workspace_size(d) <= max(16 << 20, rows * width), (rows, groups, width)


@pytest.mark.parametrize("dtype", [B.STRATA_BF16, B.STRATA_F32])
def test_more_rows_take_no_fewer_blocks(dtype):
    """A block of the backward is a row of partial sums in the workspace: as rows of a width grow its size never falls."""
    for width in list(range(1, 140)) + [203, 255, 257, 333, 501, 511, 513, 768, 999, 1024, 1293, 2048, 4096, 8192]:
        last = 0
        for rows in sorted({(1 << k) + d for k in range(0, 21) for d in (-1, 0, 1)} - {0}):
            size = B.strata_residual_norm_bwd_workspace_size(desc(rows=rows, group_rows=rows, width=width, dtype=dtype))
            assert size >= last, (width, rows)
            last = size


# ---- lists of weights ----------------------------------------------------------------

def entries(*tensors):
    """(p, g, copy, n, dtype) each."""
    return (B.ParamEntry * len(tensors))(*tensors)


def table_of(e, nbytes=None):
    L, d = B.load(), B.ParamList()
    need = L.strata_params_bytes(e, len(e))
    buf = ctypes.create_string_buffer(max(need, 1))
    st = L.strata_params_table(e, len(e), buf, need if nbytes is None else nbytes, ctypes.byref(d))
    return st, d, buf.raw


F32, BF16 = B.STRATA_F32, B.STRATA_BF16


def test_table_of_a_list():
    a = 0x100000
    e = entries((a, a + 0x40000, a + 0x80000, 4097, BF16), (a + 0x10000, None, None, 33, F32),
                (a + 0x20000, a + 0x50000, None, 1, F32), (None, None, None, 0, F32), (a + 0x30000, a + 0x60000, None, 2048, F32))
    st, d, raw = table_of(e)
    assert st == B.STRATA_OK and d.tensors == 5 and d.chunks == 5 + 0 + 1 + 0 + 2 and d.places == 4128 + 64 + 32 + 0 + 2048
    r = np.frombuffer(raw[:5 * 56], np.int64).reshape(5, 7)
    assert r[:, 0].tolist() == [a, a + 0x10000, a + 0x20000, 0, a + 0x30000] and r[:, 3].tolist() == [4097, 33, 1, 0, 2048]
    assert r[:, 1].tolist() == [a + 0x40000, 0, a + 0x50000, 0, a + 0x60000] and r[:, 2].tolist() == [a + 0x80000, 0, 0, 0, 0]
    assert r[:, 4].tolist() == [0, 4128, 4192, 4224, 4224] and r[:, 5].tolist() == [0, 5, 5, 6, 6]
    assert r[:, 6].tolist() == [1, 0, 0, 0, 0]
    assert np.frombuffer(raw[5 * 56:5 * 56 + 32], np.int32).tolist() == [0] * 5 + [2, 4, 4]


def test_lists_that_are_refused():
    L, a = B.load(), 0x100000
    good = (a, a + 0x1000, a + 0x2000, 256, F32)
    assert table_of(entries(good))[0] == B.STRATA_OK
    assert table_of(entries(good), nbytes=8)[0] == WORKSPACE
    bad = [
        [(a, a + 0x1000, None, -1, F32)], [(a, a + 0x1000, None, 1 << 40, F32)], [(None, a, None, 4, F32)],
        [(a + 4, a + 0x1000, None, 4, F32)], [(a, a + 0x1008, None, 4, F32)], [(a, a + 0x1000, a + 0x2002, 4, F32)],
        [(a, a + 0x1000, None, 4, 5)],
        [good, good],                                                   # a tensor twice
        [(a, a + 0x1000, None, 256, F32), (a + 0x3F0, None, None, 4, F32)],   # the last 4 weights again
        [(a, a, None, 4, F32)],                                         # a gradient that is the weights
        [(a, a + 0x1000, a + 0x1010, 256, F32)],                        # a copy inside the gradient
        [(a, None, a + 0x10, 8, F32)],                                  # a copy inside the weights
        [(a, a + 0x1000, a + 0x2000, 8, F32), (a + 0x3000, a + 0x1000, a + 0x2000, 8, F32)],   # one copy of two tensors
        [(a + 64 * i, 1 << 60, None, (1 << 39) + i, BF16) for i in range(3)],
    ]
    for tensors in bad:
        e = entries(*tensors)
        assert L.strata_params_bytes(e, len(e)) == 0, tensors
        assert table_of(e, 1 << 20)[0] == INVALID, tensors
    # one gradient of two tensors is only read
    assert table_of(entries((a, a + 0x1000, None, 8, F32), (a + 0x3000, a + 0x1000, None, 8, F32)))[0] == B.STRATA_OK
    assert L.strata_params_bytes(None, 1) == 0 and L.strata_params_bytes(entries(good), 0) == 0
    assert L.strata_params_table(entries(good), 1, ctypes.create_string_buffer(64), 64, None) == INVALID
    assert L.strata_params_table(entries(good), 1, None, 64, ctypes.byref(B.ParamList())) == INVALID


def plist(table=0x10000, tensors=2, chunks=5, places=8192):
    return B.ParamList(table, tensors, chunks, places)


@pytest.mark.parametrize("kw", [dict(table=None), dict(table=0x10008), dict(tensors=0), dict(chunks=-1), dict(places=-1),
                                dict(places=1 << 40), dict(chunks=1 << 31), dict(tensors=1 << 31)])
def test_lists_that_no_table_made(kw):
    L, p = B.load(), plist(**kw)
    assert L.strata_grad_norm(ref(p), 1.0, fake(), fake(), 1 << 20, None) == INVALID
    assert L.strata_grad_norm_workspace_size(ref(p)) == 0
    assert L.strata_adamw(ref(B.make_adamw_desc(1e-3, 1)), ref(p), fake(), fake(), None, None, None, None) == INVALID


def test_grad_norm_refusals():
    L, p = B.load(), plist()
    call = lambda most=1.0, norm=fake(), ws=fake(), nbytes=1 << 20, q=p: L.strata_grad_norm(ref(q), most, norm, ws, nbytes, None)  # noqa: E731
    for kw in (dict(most=0.0), dict(most=-1.0), dict(most=math.nan), dict(norm=None), dict(norm=fake(0x10004)),
               dict(ws=fake(0x10008)), dict(q=None)):
        assert call(**kw) == INVALID, kw
    assert call(ws=None) == WORKSPACE and call(nbytes=7) == WORKSPACE
    assert L.strata_grad_norm_workspace_size(ref(p)) == 256


def test_adamw_refusals():
    L, p = B.load(), plist()

    def call(kw=dict(), q=p, m=fake(), v=fake(), ms=None, vs=None, factor=None):
        d = None if kw is None else B.make_adamw_desc(**dict(dict(lr=1e-3, step=1), **kw))
        return L.strata_adamw(ref(d), ref(q), m, v, ms, vs, factor, None)
    for kw in (None, dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1),
               dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-39), dict(eps=math.inf), dict(eps=1e39),
               dict(weight_decay=-1.0), dict(weight_decay=math.inf), dict(step=0), dict(step=-3),
               dict(lr=1e38, beta1=0.99999999)):
        assert call(kw) == INVALID, kw
    for kw in (dict(q=None), dict(m=None), dict(v=None), dict(m=fake(0x10008)), dict(ms=fake()), dict(vs=fake()),
               dict(ms=fake(0x10004), vs=fake()), dict(factor=fake(0x10002))):
        assert call(**kw) == INVALID, kw
    assert call(q=plist(places=1 << 32), ms=fake(), vs=fake()) == INVALID
    # nothing to do: no launch, and so no device is needed
    assert call(q=plist(chunks=0)) == B.STRATA_OK
    assert call(q=plist(chunks=0, places=0), m=None, v=None) == B.STRATA_OK
    for n, dt, c, s, x in ((0, 1, fake(), fake(), fake()), (1 << 32, 1, fake(), fake(), fake()), (8, 2, fake(), fake(), fake()),
                           (8, 1, None, fake(), fake()), (8, 1, fake(), None, fake()), (8, 1, fake(), fake(), None),
                           (8, 0, fake(0x10004), fake(), fake())):
        assert L.strata_adamw_unpack(c, s, n, 0, x, dt, None) == INVALID


def test_binding_rejects_host_tensors():
    x = torch.zeros(4, 64)
    d = B.make_norm_desc(x)
    assert (d.rows, d.group_rows, d.width) == (4, 4, 64)
    for call in (lambda: B.strata_residual_norm(d, x, None, x, None, None, x, x),
                 lambda: B.strata_residual_norm_bwd(d, x, None, None, None, x, None, x),
                 lambda: B.make_params([x], [x]),
                 lambda: B.strata_adamw_unpack(x.byte(), x.byte(), x, False)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="2 gradients"):
        B.make_params([x], [x, x])
    with pytest.raises(ValueError, match="0 weights"):
        B.make_params([], [])
    assert B.make_norm_desc(torch.zeros(())).rows == 0 and B.make_norm_desc(torch.zeros(0, 8)).rows == 0


class OnGpu(torch.Tensor):
    """A host tensor that says it lies on GPU 0."""
    is_cuda = True
    device = property(lambda self: torch.device("cuda", 0))

    def get_device(self):
        return 0

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        with torch._C.DisableTorchFunctionSubclass():
            return func(*args, **(kwargs or {}))


def on_gpu(shape, dtype=torch.bfloat16):
    return torch.Tensor._make_subclass(OnGpu, torch.zeros(shape, dtype=dtype))


@pytest.fixture
def launches(monkeypatch):
    """The library's norm calls as a list of their names: the binding's checks alone, on tensors that need no GPU."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: made.append(name)
    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_Tensor", OnGpu)
    monkeypatch.setattr(B, "_on_gpu", lambda index, stream: None)
    return made


def norm_calls(d, shape):
    """Forward and backward of descriptor `d` with all row tensors of `shape`."""
    rows = lambda dtype=torch.bfloat16: on_gpu(shape, dtype)  # noqa: E731
    vec = lambda: on_gpu((d.rows // d.group_rows, d.width), torch.float32)  # noqa: E731
    forward = lambda **kw: B.strata_residual_norm(d, **dict(dict(  # noqa: E731
        x=rows(), gate=vec(), res=rows(), scale=vec(), shift=vec(), sum=rows(), y=rows()), **kw))
    backward = lambda **kw: B.strata_residual_norm_bwd(d, **dict(dict(  # noqa: E731
        sum=rows(), x=rows(), gate=vec(), scale=vec(), dy=rows(), dsum=rows(), dres=rows(), dx=rows(), dgate=vec(), dscale=vec(),
        dshift=vec()), **kw))
    return forward, backward


@pytest.mark.parametrize("shape", [(2, 64), (99, 64), (101, 64), (0, 64), (7, 8), (100, 32), (50, 128), (200, 32), (64,), (6400,),
                                   (3, 5, 64), (100, 8, 8), ()])
@pytest.mark.parametrize("groups", [1, 4])
def test_rows_of_another_descriptor_are_refused(shape, groups, launches):
    """All row tensors alike, but not the rows that the descriptor counts: a batch smaller than the one it was made for."""
    d = B.NormDesc(100, 100 // groups, 64, 1e-6, B.STRATA_BF16)
    for call, name in zip(norm_calls(d, shape), ("res", "sum")):
        with pytest.raises(ValueError, match=name):
            call()
    codes = dict(y=None, codes=on_gpu(shape, torch.int8), scales=on_gpu((100, 2), torch.uint8))
    with pytest.raises(ValueError, match="res"):
        norm_calls(d, shape)[0](**codes)
    assert not launches


def test_rows_of_the_descriptor_in_other_shapes(launches):
    """As many rows of its width in any shape, one another's or not."""
    d = B.NormDesc(100, 25, 64, 1e-6, B.STRATA_BF16)
    for shape, other in (((100, 64), (4, 25, 64)), ((4, 5, 5, 64), (100, 64)), ((1, 100, 64), (1, 100, 64))):
        forward, backward = norm_calls(d, shape)
        forward(x=on_gpu(other), codes=on_gpu(other, torch.int8), scales=on_gpu((200,), torch.uint8))
        backward(dy=on_gpu(other), dx=on_gpu(other))
    assert launches == ["strata_residual_norm", "strata_residual_norm_bwd"] * 3


class Learned(OnGpu):
    """Of another class than the binding's quick check knows, as nn.Parameter is."""


def test_vectors_of_a_single_group(launches):
    """[width] or [1, width], tensors and parameters alike; no other shape."""
    d = B.NormDesc(100, 100, 64, 1e-6, B.STRATA_BF16)
    forward, backward = norm_calls(d, (100, 64))
    for kind in (OnGpu, Learned):
        for shape in ((64,), (1, 64)):
            v = torch.Tensor._make_subclass(kind, torch.zeros(shape))
            forward(gate=v, scale=v, shift=v)
            backward(gate=v, scale=v)
        for shape in ((63,), (65,), (1, 63), (2, 64), (64, 1), (1, 1, 64), ()):
            v = torch.Tensor._make_subclass(kind, torch.zeros(shape))
            for call in (lambda: forward(scale=v), lambda: forward(shift=v), lambda: backward(scale=v), lambda: backward(dshift=v)):
                with pytest.raises(ValueError, match="shape"):
                    call()
        v = torch.Tensor._make_subclass(kind, torch.zeros(64, dtype=torch.bfloat16))
        with pytest.raises(ValueError, match="dtype|float32"):
            forward(scale=v)
    assert len(launches) == 8
    # of several groups: [groups, width] alone
    forward, _ = norm_calls(B.NormDesc(100, 50, 64, 1e-6, B.STRATA_BF16), (100, 64))
    for kind in (OnGpu, Learned):
        with pytest.raises(ValueError, match="scale"):
            forward(scale=torch.Tensor._make_subclass(kind, torch.zeros(64)))


def test_what_a_list_says_of_a_gradient(monkeypatch):
    """A gradient in bf16 is one, of whatever class and shape: what is wrong with it is named."""
    w = torch.Tensor._make_subclass(OnGpu, torch.zeros(4, 8))
    for dtype in (torch.bfloat16, torch.float32):
        with pytest.raises(ValueError, match="shape"):
            B.make_params([w], [on_gpu((4, 7), dtype)])
    with pytest.raises(ValueError, match="dtype"):
        B.make_params([w], [on_gpu((4, 8), torch.float16)])
    monkeypatch.setattr(B, "load", lambda: (_ for _ in ()).throw(RuntimeError("the list was accepted")))
    with pytest.raises(RuntimeError, match="accepted"):
        B.make_params([w], [on_gpu((4, 8))])


# ---- the oracle ------------------------------------------------------------------------

@pytest.mark.parametrize("second", [False, True])
def test_oracle_codes(second):
    """Every code of every scale that states can have is a value that encodes to itself with the number 0, but where
    its group's largest is 15 of 8 steps, which belongs to the next scale."""
    u = T.UNIT[second]
    top = 127 if not second else 255
    for e in (u + 1, u + 2, 60, 100, 127, 200, 253, 254):
        codes = np.arange(256, dtype=np.uint8).reshape(-1, 32).copy()
        codes[:, 0] = top - 1                                   # 14 eighths of the group's power of two
        codes[(codes & 127 if not second else codes) == top] = 0
        codes = codes.reshape(-1)
        v = T.decode(codes, np.full(8, e), second)
        assert np.array_equal(v.astype(np.float32), v)
        c, s = T.encode(v, np.zeros(256), second)
        assert (s == e).all()
        same = codes == c
        assert (same | (codes == 128)).all()                    # -0 is 0
        assert (np.diff(T.decode(np.arange(top + 1), np.full((top + 32) // 32, e), second)) > 0).all()


@pytest.mark.parametrize("second", [False, True])
def test_oracle_rounding_is_unbiased(second):
    """The mean over all random numbers k 2^-16 is the value to 2^-16 steps and the rounding of a sum below 16, 2^-21
    steps: with f the value's distance to the lower code, floor(2^16 f) of the 2^16 numbers reach over the border."""
    x = np.float32([1.0, 0.7312, 0.5001, 0.1234, 0.01, 3.1e-4, 7.7e-6] + [0.0] * 25)
    if not second:
        x[1::2] *= -1
    r = (np.arange(1 << 16) / 65536).astype(np.float32)
    c, s = T.encode(np.tile(x, 1 << 16), np.repeat(r, 32), second)
    mean = T.decode(c, s, second).reshape(-1, 32).mean(0)
    step = np.maximum(2.0 ** (np.floor(np.log2(np.abs(x) + 1e-30)) - 3), 2.0 ** (-T.UNIT[second]))
    assert (np.abs(mean - x) <= step * (2.0 ** -16 + 2.0 ** -20))[:7].all() and (mean[7:] == 0).all()


def test_oracle_gradient_by_differences():
    g = np.random.default_rng(3)
    res, x, dy, dsum = (g.normal(size=(2, 3, 5)) for _ in range(4))
    gate, scale, shift = (g.normal(size=(2, 5)) for _ in range(3))

    def loss(res, x, gate, scale, shift):
        s = T.add(res, x, gate)
        return (T.norm(s, scale, shift)[0] * dy).sum() + (s * dsum).sum()
    out = T.norm_backward(T.add(res, x, gate), dy, dsum, x, gate, scale)
    for i, name in enumerate(("dres", "dx", "dgate", "dscale", "dshift")):
        args = [res, x, gate, scale, shift]
        for at in np.ndindex(args[i].shape):
            d = np.zeros_like(args[i])
            d[at] = 1e-5
            up, down = (loss(*(a + f * d if k == i else a for k, a in enumerate(args))) for f in (1, -1))
            assert abs((up - down) / 2e-5 - out[name][at]) < 1e-7, (name, at)


def test_oracle_adamw_is_the_sum_it_stands_for():
    """From zero states m and v are weighted means of the gradients, and the first step is lr times their sign."""
    g = np.random.default_rng(4).normal(size=(6, 9))
    p, m, v = np.ones(9), np.zeros(9), np.zeros(9)
    for k in range(6):
        was = p
        p, m, v = T.adamw(p, g[k], m, v, 1e-2, k + 1, 0.9, 0.99, 1e-12, 0.0)
        if k == 0:
            assert np.allclose(was - p, 1e-2 * np.sign(g[0]), rtol=1e-9)
    w = 0.9 ** np.arange(5, -1, -1) * 0.1
    assert np.allclose(m, (w[:, None] * g).sum(0), rtol=1e-12)
    w = 0.99 ** np.arange(5, -1, -1) * 0.01
    assert np.allclose(v, (w[:, None] * g * g).sum(0), rtol=1e-12)


def test_oracle_random_numbers_are_even():
    """65536 places: mean and variance of 16 uniform bits within 5 deviations, for both numbers, and no correlation."""
    a, b = T.random_numbers(1234567890123, np.arange(65536))
    for x in (a, b):
        assert abs(x.mean(dtype=np.float64) - 0.5) < 5 / 12 ** 0.5 / 256
        assert abs(x.var(dtype=np.float64) * 12 - 1) < 5 * 0.9 / 256
    assert abs(np.corrcoef(a, b)[0, 1]) < 5 / 256 and abs(np.corrcoef(a[1:], a[:-1])[0, 1]) < 5 / 256
    assert not np.array_equal(a, T.random_numbers(1234567890124, np.arange(65536))[0])


def test_codes_of_the_norm_use_the_rows_form():
    """The 8-bit output's rule is that of activations."""
    x = np.random.default_rng(5).normal(size=64)
    c, s = R.encode(x)
    assert np.abs(R.decode(c, s) - x).max() <= 2.0 ** (s.max() - 134.0)
