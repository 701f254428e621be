"""What a block's saved state says about its lse and output, without a GPU."""
import pytest
import torch

from paper_2606_31248_amd import binding as B
from paper_2606_31248_amd import pipeline


def saved(**kw):
    d = B.make_qkv_desc(1, 2, 1, 1, 1, 64, B.STRATA_BF16)
    return pipeline.BlockSaved(**dict(dict(qkv=d, window=(1, 1, 1), scale=0.125, wq=None, wk=None, cs=None,
                                           lse=torch.zeros(1, 2, 1, 1, 1), rows=torch.zeros(1, 1, 1, 1, d.row_stride),
                                           out=torch.zeros(1, 2, 1, 1, 1, 64)), **kw))


@pytest.mark.parametrize("name", ["qkv", "window", "scale", "wq", "wk", "cs", "rows"])
def test_a_field_that_shapes_the_attention(name):
    s = saved()
    assert not s.again
    setattr(s, name, getattr(s, name))
    assert s.again


def test_the_forwards_own_state():
    s = saved()
    s.out, s.lse, s.gate = s.out.clone(), s.lse.clone(), None      # moved away and back
    assert not s.again and saved(again=True).again
