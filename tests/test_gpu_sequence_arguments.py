"""Numbers that the calls around the decode step take: what a descriptor's field
does not hold is refused, not cut; and streams by their number."""
import pytest
import torch

from paper_2609_38169_amd import stepq
from _sequence import tokens
from test_gpu_prefix_attention import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("python", [False, True])
@pytest.mark.parametrize("rule", [1 << 32, (1 << 32) + 1, -(1 << 32), 0.5])
def test_rules_that_are_none(rule, python, monkeypatch):
    if python:
        monkeypatch.setattr(stepq, "_native", stepq._PythonChecks)
    x = [t.to(DEV) for t in tokens(8, 2, 1, 64, 64, torch.bfloat16, torch.float32, 1)]
    o, S = torch.empty((8, 2, 64), dtype=torch.bfloat16, device=DEV), torch.empty((8, 2, 64, 64), device=DEV)
    cu = torch.arange(9, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        stepq.stepq_prompt(*x, o, S, rule, cu_seqlens=cu)
    with pytest.raises(ValueError):
        stepq.stepq_state_step(S, cu[:8], *x, torch.empty((8, 2, 64), device=DEV), rule)


@pytest.mark.parametrize("prefix", [40.5, 1 << 63, -0.5])
def test_prefix_lengths_that_are_none(prefix):
    q, k, v, pre, _, table, lengths = (t.to(DEV) if isinstance(t, torch.Tensor) else t
                                       for t in inputs(2, 4, 2, 64, 40, [5, 6], 16, torch.bfloat16))
    with pytest.raises(ValueError):
        stepq.stepq_prefix_attention(q, k, v, pre, prefix, table, lengths, torch.empty_like(q))


def test_whole_numbers_of_any_type():
    x = inputs(2, 4, 2, 64, 40, [5, 6], 16, torch.bfloat16)
    got = []
    for prefix in (40, 40.0, torch.tensor(40)):
        q, k, v, pre, _, table, lengths = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in x)
        o = torch.empty_like(q)
        stepq.stepq_prefix_attention(q, k, v, pre, prefix, table, lengths, o)
        got.append(o)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_the_default_stream_by_its_number():
    x = [t.to(DEV) for t in tokens(100, 2, 1, 64, 64, torch.bfloat16, torch.float32, 1)]
    y = inputs(2, 4, 2, 64, 40, [5, 6], 16, torch.bfloat16)
    y = [t.to(DEV) if isinstance(t, torch.Tensor) else t for t in y]
    got = []
    for kw in ({}, dict(stream=0)):
        o, S = torch.empty((100, 2, 64), dtype=torch.bfloat16, device=DEV), torch.empty((1, 2, 64, 64), device=DEV)
        a = torch.empty_like(y[0])
        stepq.stepq_prompt(*x, o, S, **kw)
        stepq.stepq_prefix_attention(*y, a, **kw)
        torch.cuda.synchronize()
        got.append((o, S, a))
    assert all(torch.equal(p, q) for p, q in zip(*got))
