"""Bounds of packed prompts that start past the first token or are malformed:
what lies in no sequence is not touched, and what lies in one is what it would
be by itself, whichever way the call walks it."""
import pytest
import torch

from paper_2609_38169_amd import stepq
from _sequence import DECAY, DELTA, tokens
from test_gpu_prompt import close_f32, close_o, recurrence

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def call(x, cu, rule, start=None):
    T, hv, dv = x[2].shape
    n, dk = len(cu) - 1, x[0].shape[2]
    o, out = torch.full((T, hv, dv), 7.0, dtype=x[2].dtype, device=DEV), torch.full((n, hv, dk, dv), 7.0, device=DEV)
    stepq.stepq_prompt(*(t.to(DEV) for t in x), o, out, rule, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device=DEV),
                       state_in=None if start is None else start.to(DEV))
    torch.cuda.synchronize()
    return o.cpu(), out.cpu()


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("hv", [1, 200], ids=["segments", "whole"])
@pytest.mark.parametrize("cu", [[1000, 1000, 1700], [900, 1700], [64, 65, 1700], [0, 1000, 1000]], ids=str)
def test_sequences_that_start_later(cu, hv, act, rule):
    """A first sequence past the first token, empty or not; 1 head goes in segments, 200 heads do not."""
    if hv > 1:
        cu = [c // 10 for c in cu]
    T = 1700 if hv == 1 else 170
    x = tokens(T, hv, hv, 64, 64, act, F32, 3, low=0.98)
    n = len(cu) - 1
    start = 0.3 * torch.randn((n, hv, 64, 64), generator=torch.Generator().manual_seed(4))
    o, out = call(x, cu, rule, start)
    assert (o[:cu[0]] == 7.0).all() and (o[cu[-1]:] == 7.0).all()
    for i in range(n):
        t = slice(cu[i], cu[i + 1])
        ro, rs = recurrence(*(y[t] for y in x), start[i], rule)
        if cu[i] == cu[i + 1]:
            assert torch.equal(out[i], start[i])
        else:
            close_o(o[t], ro, f"o of sequence {i}")
            close_f32(out[i], rs, f"state of sequence {i}")


@pytest.mark.parametrize("rule", [DECAY, DELTA])
def test_malformed_bounds_leave_the_others_right(rule):
    """Bounds that go down give an empty sequence, ones past the tokens are cut; the sequences that are well
    formed are what they are in a call of their own."""
    x = tokens(100, 1, 1, 64, 64, BF16, F32, 2)
    o, out = call(x, [0, 40, 30, 5000], rule)
    ro, rs = recurrence(*(y[:40] for y in x), torch.zeros(1, 64, 64), rule)
    close_f32(out[0], rs, "state of sequence 0")
    assert not out[1].any()
    close_o(o[:30], ro[:30], "o of the tokens of sequence 0 alone")
    ro, rs = recurrence(*(y[30:] for y in x), torch.zeros(1, 64, 64), rule)
    close_o(o[40:], ro[10:], "o of the tokens of sequence 2 alone")
    close_f32(out[2], rs, "state of sequence 2")
