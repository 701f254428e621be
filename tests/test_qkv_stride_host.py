"""The 8-bit call has no rows and does not compute with their stride: any value is one to a machine without a GPU,
where the launch is refused by the runtime (the sanitizers watch the host code up to there)."""
import ctypes

import pytest
import torch

from paper_2606_31248_amd import binding as B


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: never launched on a GPU")
@pytest.mark.parametrize("stride", [0, -8, 3, (1 << 62) + 64, -(1 << 62), (1 << 63) - 1])
def test_any_row_stride(stride):
    d = B.make_qkv_desc(2, 4, 3, 5, 7, 64, B.STRATA_BF16, kv_heads=2, gate_dim=64, row_stride=stride)
    p = ctypes.c_void_p(0x10000)
    assert B.load().strata_qkv_heads_ckpt(ctypes.byref(d), p, p, None, None, None, p, p, p, p, None) == B.STRATA_ERR_HIP
