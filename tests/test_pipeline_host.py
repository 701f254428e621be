"""What a block's saved state says about its lse and output, and what an optimiser counts, without a GPU."""
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


class Host:
    """The binding's calls on host tensors: lists that are only kept, steps that are recorded and, if told to, refused."""

    def __init__(self, monkeypatch):
        self.steps, self.refuse = [], False
        for name in ("make_params", "strata_grad_norm_workspace_size", "strata_grad_norm", "strata_adamw"):
            monkeypatch.setattr(B, name, getattr(self, name))
        monkeypatch.setattr(pipeline, "_current_stream", lambda device: 0, raising=False)
        monkeypatch.setattr(B, "_on_gpu", lambda index, stream: 0)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)

    def make_params(self, p, g, copies=None):
        made = B.Params((list(p), list(g), copies), B.ParamList(0, len(p), len(p), 32 * len(p)),
                        torch.zeros(1, dtype=torch.uint8), [32 * i for i in range(len(p))], torch.device("cpu"))
        return made

    def strata_grad_norm_workspace_size(self, params):
        return 0

    def strata_grad_norm(self, params, max_norm, norm, ws):
        pass

    def strata_adamw(self, desc, params, *states):
        if self.refuse:
            raise B.StrataError(B.STRATA_ERR_INVALID_ARG, "refused")
        self.steps.append((desc.step, desc.seed, params.tensors[1]))


def test_a_refused_step_is_not_counted(monkeypatch):
    host = Host(monkeypatch)
    opt = pipeline.AdamW([torch.zeros(4)], [torch.zeros(4)], seed=3, max_norm=1.0)
    opt.step(1e-3)
    host.refuse = True
    with pytest.raises(B.StrataError):
        opt.step(-1.0)
    assert opt.steps == 1
    host.refuse = False
    opt.step(1e-3)
    assert opt.steps == 2 and [k for k, _, _ in host.steps] == [1, 2] and host.steps[0][1] != host.steps[1][1]


def loss(p, k):
    return sum(((i + k) * w).sum() for i, w in enumerate(p))


def test_gradients_allocated_anew(monkeypatch):
    """A loop whose zero_grad sets gradients to None: a step on the list's old ones is refused, and none is counted;
    renew takes the new ones and keeps states and steps."""
    host = Host(monkeypatch)
    p = [torch.nn.Parameter(torch.ones(4)) for _ in range(3)]
    loss(p, 1).backward()
    opt = pipeline.AdamW(p, [w.grad for w in p], seed=5)
    states = opt.m, opt.v
    opt.step(1e-3)
    loss(p, 1).backward()                      # added in place: the same tensors
    opt.step(1e-3)
    for fresh in (False, True):                # set to None and not computed again; computed again
        for w in p:
            w.grad = None
        if fresh:
            loss(p, 2).backward()
        with pytest.raises(ValueError, match="renew"):
            opt.step(1e-3)
    assert opt.steps == 2 and len(host.steps) == 2
    opt.renew([w.grad for w in p])
    opt.step(1e-3)
    assert opt.steps == 3 and opt.m is states[0] and opt.v is states[1] and opt.params.tensors[0] == p
    assert all(a is w.grad for a, w in zip(host.steps[2][2], p)) and [k for k, _, _ in host.steps] == [1, 2, 3]
    # gradients that are not the weights' own are the caller's to fill
    mine = [torch.zeros(4) for _ in p]
    opt.renew(mine)
    p[0].grad = None
    opt.step(1e-3)
    assert host.steps[3][2] == mine
    # one without a gradient this time
    opt.renew([mine[0], None, mine[2]], copies=[None] * 3)
    opt.step(1e-3)
    assert host.steps[4][2][1] is None and opt.steps == 5


def test_a_list_that_is_refused_leaves_the_old_one(monkeypatch):
    host = Host(monkeypatch)
    g = [torch.zeros(4)]
    opt = pipeline.AdamW([torch.zeros(4)], g)
    old = opt.params

    def refuse(*args):
        raise ValueError("refused")
    monkeypatch.setattr(B, "make_params", refuse)
    with pytest.raises(ValueError, match="refused"):
        opt.renew([torch.zeros(5)])
    assert opt.params is old
    opt.step(1e-3)
    assert host.steps[0][2] == g


def test_gradients_that_another_stream_still_reads(monkeypatch):
    """What renew lets go is marked for the streams that steps ran on beside the list's own, and only then."""
    host, now, marked = Host(monkeypatch), [0], []
    monkeypatch.setattr(B, "_on_gpu", lambda index, stream: now[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: now[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: marked.append((t, s)))
    first, second, third = ([torch.zeros(4), None] for _ in range(3))
    opt = pipeline.AdamW([torch.zeros(4), torch.zeros(2)], first, [None, torch.zeros(2, dtype=torch.bfloat16)])
    copy = opt.params.tensors[2][1]
    opt.step(1e-3)
    opt.renew(second)
    assert not marked
    table = opt.params.table
    now[0] = 5
    opt.step(1e-3), opt.step(1e-3)
    assert marked and all(s == 5 for _, s in marked) and any(t is table for t, _ in marked)
    now[0] = 0
    marked.clear()
    opt.renew(third)
    assert [s for _, s in marked] == [5, 5] and marked[0][0] is second[0] and marked[1][0] is copy
    marked.clear()
    opt.step(1e-3)
    opt.renew(first)
    assert not marked and len(host.steps) == 4
