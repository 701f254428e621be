"""Refusals of the projection-row and 8-bit entry points that need no GPU: the C ABI
rejects bad arguments before any launch, the binding host tensors."""
import ctypes

import pytest
import torch

from paper_2606_31248_amd import binding as B

GOOD = dict(B=2, heads=4, Z=3, H=5, W=7, head_dim=64, dtype=B.STRATA_BF16, kv_heads=2, gate_dim=64)
INVALID, UNSUPPORTED, WORKSPACE = B.STRATA_ERR_INVALID_ARG, B.STRATA_ERR_UNSUPPORTED, B.STRATA_ERR_WORKSPACE


def desc(**kw):
    return B.make_qkv_desc(**dict(GOOD, **kw))


def fake(addr=0x10000):
    return ctypes.c_void_p(addr)


def ref(d):
    return None if d is None else ctypes.byref(d)


def fwd(d, rows=fake(), wq=None, wk=None, cs=None, q=fake(), k=fake(), v=fake(), gate=fake(), codes=None, scales=None):
    return B.load().strata_qkv_heads(ref(d), rows, wq, wk, cs, q, k, v, gate, codes, scales, None)


def again(d, codes=fake(), scales=fake(), q=fake(), gate=fake(), wq=None):
    return B.load().strata_qkv_heads_ckpt(ref(d), codes, scales, wq, None, None, q, fake(), fake(), gate, None)


def bwd(d, rows=fake(), codes=None, scales=None, wq=fake(), wk=fake(), dq=fake(), dgate=fake(), drows=fake(),
        dwq=fake(), dwk=fake(), ws=fake(), nbytes=1 << 40):
    return B.load().strata_qkv_heads_bwd(ref(d), rows, codes, scales, wq, wk, None, dq, fake(), fake(), dgate, drows,
                                         dwq, dwk, ws, nbytes, None)


BAD = [
    (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID), (dict(kv_heads=8), INVALID),
    (dict(Z=0), INVALID), (dict(W=-1), INVALID), (dict(gate_dim=2), INVALID), (dict(gate_dim=32), INVALID),
    (dict(dtype=2), INVALID), (dict(head_dim=48, gate_dim=0), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(B=1 << 20, H=1 << 4, W=1 << 4), INVALID),                              # 2^28 tokens and more
    (dict(B=1 << 30, Z=1 << 30, H=1 << 30, W=1 << 30), INVALID),                 # beyond 64 bits if multiplied out
    (dict(heads=40000, kv_heads=40000), INVALID),                                # 65535 heads in a row
]


@pytest.mark.parametrize("kw,status", BAD)
def test_every_call_rejects_a_bad_descriptor(kw, status):
    d = desc(**kw)
    assert fwd(d) == status and B.load().strata_last_error() != b""
    assert again(d) == status
    assert bwd(d) == status
    assert B.strata_qkv_heads_bwd_workspace_size(d) == 0


def test_eps_is_not_read_without_the_norm():
    assert fwd(desc(qk_norm=False, eps=-1.0), rows=None) == INVALID
    assert b"rows: null" in B.load().strata_last_error()   # past the descriptor


@pytest.mark.parametrize("stride", [511, 767, 772, 0, -8, 1 << 62])
def test_row_stride_rules(stride):
    d = desc(row_stride=stride)   # width (4 + 2 + 2 + 4) 64 = 768
    assert d.width == 768 and d.kept == 768
    assert fwd(d) == INVALID and bwd(d) == INVALID
    # the 8-bit form has no row stride
    assert again(d, codes=None) == INVALID and b"codes" in B.load().strata_last_error()


def test_forward_pointers():
    d, plain = desc(), desc(gate_dim=0)
    assert fwd(None) == INVALID
    for kw in (dict(rows=None), dict(q=None), dict(k=None), dict(v=None), dict(gate=None), dict(rows=fake(0x10008)),
               dict(q=fake(0x10004)), dict(gate=fake(0x10002)), dict(cs=fake(0x10008)), dict(wq=fake()), dict(wk=fake()),
               dict(wq=fake(), wk=fake(0x10004)), dict(codes=fake()), dict(scales=fake()),
               dict(codes=fake(0x10008), scales=fake()), dict(codes=fake(), scales=fake(0x10001))):
        assert fwd(d, **kw) == INVALID, kw
    assert fwd(plain) == INVALID and b"gate" in B.load().strata_last_error()      # a gate that the rows do not hold
    assert fwd(desc(qk_norm=False), wq=fake(), wk=fake()) == INVALID              # a scale without a norm


def test_again_pointers():
    d = desc()
    for kw in (dict(codes=None), dict(scales=None), dict(q=None), dict(gate=None), dict(codes=fake(0x10008)),
               dict(wq=fake()), dict(gate=fake(0x10004))):
        assert again(d, **kw) == INVALID, kw
    # one-per-head gate logits are not in the 8-bit form
    assert again(desc(gate_dim=1)) == INVALID and again(desc(gate_dim=0)) == INVALID


def test_backward_pointers_and_workspace():
    d = desc()
    for kw in (dict(rows=None), dict(codes=fake(), scales=fake()), dict(rows=None, codes=fake()),
               dict(rows=None, scales=fake()), dict(dq=None), dict(drows=None), dict(dgate=None), dict(dwq=None),
               dict(dwk=None), dict(wq=None), dict(wq=None, wk=None), dict(drows=fake(0x10008)),
               dict(dwq=fake(0x10004)), dict(ws=fake(0x10008))):
        assert bwd(d, **kw) == INVALID, kw
    need = B.strata_qkv_heads_bwd_workspace_size(d)
    assert need > 0 and need % 256 == 0
    assert bwd(d, ws=None) == WORKSPACE and bwd(d, nbytes=255) == WORKSPACE
    assert bwd(desc(gate_dim=0)) == INVALID                                        # dgate without a gate
    assert B.strata_qkv_heads_bwd_workspace_size(desc(qk_norm=False)) == 0


def test_workspace_stays_small():
    """The partial weight gradients: 5 MiB, or 5 % of dq, dk and dv where that is more."""
    for kw in (dict(), dict(B=1, Z=1, H=1, W=1), dict(B=16, heads=16, kv_heads=16, Z=8, H=64, W=64),
               dict(B=1, heads=1, kv_heads=1, head_dim=128, gate_dim=128, Z=24, H=64, W=64),
               dict(B=81, heads=16, kv_heads=1, Z=24, H=64, W=64, head_dim=32, gate_dim=1),
               dict(B=24, heads=16, kv_heads=4, Z=24, H=16, W=16, gate_dim=1)):
        d = desc(**kw)
        grads = 2 * d.B * d.Z * d.H * d.W * 3 * d.heads * d.head_dim
        assert 0 < B.strata_qkv_heads_bwd_workspace_size(d) <= max(5 << 20, 0.05 * grads)


@pytest.mark.parametrize("n,dtype,x,codes,scales", [
    (0, 1, fake(), fake(), fake()), (-1, 1, fake(), fake(), fake()), (1 << 40, 1, fake(), fake(), fake()),
    (8, 3, fake(), fake(), fake()), (8, 1, None, fake(), fake()), (8, 1, fake(), None, fake()),
    (8, 1, fake(), fake(), None), (8, 1, fake(0x10008), fake(), fake()), (8, 0, fake(), fake(0x10008), fake()),
    (8, 0, fake(), fake(), fake(0x10001)),
])
def test_ckpt_rules(n, dtype, x, codes, scales):
    L = B.load()
    assert L.strata_ckpt_pack(x, n, codes, scales, dtype, None) == INVALID
    assert L.strata_ckpt_unpack(codes, scales, n, x, dtype, None) == INVALID


def test_binding_rejects_host_tensors():
    d = desc(B=1, Z=1, H=1, W=1)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    h, rows = bf(1, 4, 1, 1, 1, 64), bf(1, 1, 1, 1, 768)
    codes, scales = torch.zeros(768, dtype=torch.int8), torch.zeros(24, dtype=torch.uint8)
    for call in (lambda: B.strata_qkv_heads(d, rows, None, None, None, h, h, h, h),
                 lambda: B.strata_qkv_heads_ckpt(d, codes, scales, None, None, None, h, h, h, h),
                 lambda: B.strata_qkv_heads_bwd(d, rows, None, None, None, None, None, h, h, h, h, rows, None, None, None),
                 lambda: B.strata_ckpt_pack(rows, codes, scales),
                 lambda: B.strata_ckpt_unpack(codes, scales, rows)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="torch.Tensor"):
        B.strata_ckpt_pack(0x1000, codes, scales)
    with pytest.raises(ValueError, match="rows"):
        B.strata_qkv_heads(d, None, None, None, None, h, h, h, h)
