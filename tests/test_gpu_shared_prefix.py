"""The shared-prefix example: prompts, states, pool and attention together,
against the same stack token by token in 64 bits.

Tolerances.  float32 without the pool: each call's own error is below 2e-5 of
its outputs' scale and the projections' below 128 x 2^-24 of theirs; 4 layers
carry them on with gains of a few: 1e-3 of the largest output.  With the pool:
the states are kept in 8 bits, half a step of 1/127 of a tile's largest
elements per element, which o, a sum of d products with |q| = 1, passes on as a
part in 254 at most of a state row's norm each; two such layers, and the layers
after them: 5 % of the largest output (and more than 0: the pool is used)."""
import importlib.util
import os

import pytest
import torch

from _sequence import recurrence, DECAY, DELTA

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("shared_prefix", os.path.join(ROOT, "examples", "shared_prefix.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def whole(stack, x):
    """All tokens of one request through the stack, in float64 on the CPU."""
    x = x.cpu().double()
    n = x.shape[0]
    for i, kind in enumerate(stack.kinds):
        w_in, w_out, w_gate = (w[i].cpu().double() for w in (stack.w_in, stack.w_out, stack.w_gate))
        y = x * torch.rsqrt((x ** 2).mean(-1, keepdim=True) + 1e-6)
        q, k, v = (y @ w_in).split(stack.widths(kind), -1)[:3]
        if kind == "attention":
            q, k, v = (z.reshape(n, -1, stack.head_dim) for z in (q, k, v))
            rep = stack.q_heads // stack.kv_heads
            k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
            s = torch.einsum("thd,uhd->htu", q, k) * stack.head_dim ** -0.5
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), float("-inf"))
            o = torch.einsum("htu,uhd->thd", torch.softmax(s, -1), v)
        else:
            q, k, v = (z.reshape(n, -1, stack.d) for z in (q, k, v))
            q, k = (z / z.norm(dim=-1, keepdim=True) for z in (q, k))
            a, b = (y @ w_gate).split(stack.v_heads, -1)
            S = torch.zeros((stack.v_heads, stack.d, stack.d), dtype=torch.float64)
            o, _ = recurrence(q, k, v, torch.sigmoid(a + 4), torch.sigmoid(b), S, DELTA if kind == "delta" else DECAY)
        x = x + o.reshape(n, -1) @ w_out
    return x


@pytest.mark.parametrize("quantized,tol", [(False, 1e-3), (True, 5e-2)])
def test_requests_over_a_shared_prefix(quantized, tol):
    m = example()
    stack = m.Stack(kinds=("delta", "decay", "attention", "delta"), width=128, v_heads=4, qk_heads=2, d=64, q_heads=8,
                    kv_heads=2, head_dim=64, dtype=torch.float32)
    g = torch.Generator().manual_seed(3)
    draw = lambda n: torch.randn((n, stack.width), generator=g)
    P, lens, steps = 150, [1, 70, 13], 3
    prefix, prompts, more = draw(P), [draw(n) for n in lens], [draw(len(lens)) for _ in range(steps)]
    server = m.Server(stack, prefix.cuda(), len(lens), 80, page=16, quantized=quantized)
    got = [server.admit([p.cuda() for p in prompts])] + [server.step(x.cuda()) for x in more]
    got = torch.stack([x.cpu().double() for x in got], 1)                     # [B][1 + steps][width]
    worst = 0.0
    for b, p in enumerate(prompts):
        want = whole(stack, torch.cat([prefix, p] + [x[b:b + 1] for x in more]))[-1 - steps:]
        worst = max(worst, float((got[b] - want).abs().max() / want.abs().max()))
        first = float((got[b, 0] - want[0]).abs().max() / want.abs().max())
        assert first <= 1e-3, (b, first)                                      # no pool before the first step
    assert worst <= tol, worst
    assert not quantized or worst > 1e-5
