"""The workspace of the rows' backward to the byte: what strata_qkv_heads_bwd_workspace_size says and not one less."""
import ctypes

import pytest

from paper_2606_31248_amd import binding as B


@pytest.mark.parametrize("kw", [dict(), dict(head_dim=32, gate_dim=1), dict(head_dim=128, gate_dim=0), dict(kv_heads=4),
                                dict(B=1, Z=24, H=64, W=43, heads=1, kv_heads=1, head_dim=128, gate_dim=0),
                                dict(B=16, Z=8, H=64, W=64, heads=16, kv_heads=16), dict(row_stride=776)])
def test_one_byte_short(kw):
    d = B.make_qkv_desc(**dict(dict(B=2, heads=4, Z=3, H=5, W=7, head_dim=64, dtype=B.STRATA_BF16, kv_heads=2, gate_dim=64), **kw))
    p, need = ctypes.c_void_p(0x10000), B.strata_qkv_heads_bwd_workspace_size(d)
    call = lambda n: B.load().strata_qkv_heads_bwd(ctypes.byref(d), p, None, None, p, p, None, p, p, p, p if d.gate_dim else None,  # noqa: E731
                                                   p, p, p, p, n, None)
    assert need >= 2 * d.head_dim * 4
    assert call(need - 1) == B.STRATA_ERR_WORKSPACE and call(0) == B.STRATA_ERR_WORKSPACE
    assert str(need).encode() in B.load().strata_last_error()
