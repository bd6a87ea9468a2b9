"""Prompts whose tokens differ in size by many powers of two: each token's output
is right beside the terms it is itself the sum of, whatever else its chunk holds.

Tolerances.  With L the gates' quotients, P = L (Q K^T), M = strict lower part of
beta L (K K^T), T = (I + M)^-1 and R = V - G K S (Delta), an output is
G q S + P T beta R.  Each factor is formed from operands of 22 bits or more and
summed in fp32 over d_k or 64 terms: (128 + 3 x 64) 2^-24 = 1.9e-5 at the worst,
with the gates' 2^-20 taken as 3e-5, of the sum of the terms' magnitudes
  G |q| |S| + |P| |T| |I + M| |T| beta (|V| + G |K| |S|)
(a computed inverse is off by such a part of |T| |I + M| |T|; the decay rule has
T = I, M = 0).  It is formed here in 64 bits, token by token; nothing in it
comes from later tokens.  A bfloat16 output is rounded once more, by up to 2^-8
of itself.  The final state, G S + (w K)^T T beta R with w the gates from each
token to the end, the same way."""
import pytest
import torch

from paper_2609_38169_amd import stepq
from _sequence import DECAY, DELTA, recurrence, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def magnitude(q, k, v, alpha, beta, S, rule):
    """The sums above for up to 64 tokens of one sequence: outputs' [T][Hv][dv] and the state's, float64."""
    q, k, v, alpha, beta, S = (x.double() for x in (q, k, v, alpha, beta, S))
    rep = v.shape[1] // q.shape[1]
    q, k = (x.repeat_interleave(rep, 1).transpose(0, 1) for x in (q, k))                    # [Hv][T][dk]
    v, beta, G = v.transpose(0, 1), beta.t()[..., None], torch.cumsum(torch.log(alpha), 0).t()
    L = torch.exp(G[:, :, None] - G[:, None, :]).tril()
    G = torch.exp(G)[..., None]
    P = ((q @ k.transpose(1, 2)) * L).abs()
    R = v.abs() * beta
    if rule == DELTA:
        M = (beta * (k @ k.transpose(1, 2)) * L).tril(-1)
        eye = torch.eye(M.shape[-1], dtype=torch.float64)
        T = torch.linalg.solve_triangular(eye + M, eye.expand_as(M), upper=False, unitriangular=True).abs()
        R = T @ ((eye + M).abs() @ (T @ (beta * (v.abs() + G * (k.abs() @ S.abs())))))
    w = L[:, -1, :, None]
    return (G * (q.abs() @ S.abs()) + P @ R).transpose(0, 1), G[:, -1:] * S.abs() + (k.abs() * w).transpose(1, 2) @ R


def check(x, rule, gate=F32, seed=0):
    q, k, v, alpha, beta = x
    T, hv, dv = v.shape
    dk = q.shape[2]
    assert T <= 64
    S = 0.3 * torch.randn((1, hv, dk, dv), generator=torch.Generator().manual_seed(seed))
    o, out = torch.full((T, hv, dv), 7.0, dtype=v.dtype, device=DEV), torch.empty((1, hv, dk, dv), device=DEV)
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    stepq.stepq_prompt(*(t.to(DEV) for t in x), o, out, rule, cu_seqlens=cu, state_in=S.to(DEV))
    torch.cuda.synchronize()
    ro, rs = recurrence(q, k, v, alpha, beta, S[0], rule)
    mo, ms = magnitude(q, k, v, alpha, beta, S[0], rule)
    off = (o.cpu().double() - ro).abs()
    worst = (off / (3e-5 * mo + (0 if v.dtype == F32 else 2.0 ** -8) * ro.abs() + 1e-300)).amax(dim=(1, 2))
    assert (worst <= 1).all(), (int(worst.argmax()), float(worst.max()))
    worst = ((out[0].cpu().double() - rs).abs() / (3e-5 * ms + 1e-300)).max()
    assert worst <= 1, float(worst)


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("what", ["k", "q", "v"])
@pytest.mark.parametrize("power", [12, 20, 28, 32])
@pytest.mark.parametrize("dk,dv", [(128, 128), (77, 64)])
def test_one_large_token(dk, dv, power, what, act, rule):
    """A token far larger than those before it leaves them what they are."""
    x = tokens(64, 2, 1, dk, dv, act, F32, 5)
    dict(zip("qkv", x))[what][60] *= 2.0 ** power
    check(x, rule)


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
def test_one_large_value(act, rule):
    """A single entry: its token's other columns and its column's other tokens stay."""
    x = tokens(64, 2, 2, 64, 64, act, F32, 6)
    x[2][60, 1, 5] *= 2.0 ** 32
    check(x, rule)


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_tokens_of_every_size(seed, act, rule):
    """Norms of q, k and v from 2^-20 to 2^20 of one another (the Delta rule's keys up to 1) in one chunk."""
    x = tokens(64, 2, 1, 128, 128, act, F32, seed)
    g = torch.Generator().manual_seed(seed + 100)
    for t, top in zip(x, (20, 0 if rule == DELTA else 20, 20)):
        t *= (2.0 ** torch.randint(-20, top + 1, (64, 1, 1), generator=g)).to(act)
    check(x, rule)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("norm,T", [(1.5, 64), (2.0, 64), (4.0, 40), (8.0, 20)])
def test_keys_longer_than_one(norm, T, act):
    """beta |k|^2 beyond 2: the recurrence itself grows from token to token, and the first ones stay as they are."""
    x = tokens(T, 2, 1, 64, 64, act, F32, 8)
    x[1].mul_(norm)
    check(x, DELTA)


@pytest.mark.parametrize("act", [F32, BF16])
def test_equal_keys_of_norm_two(act):
    x = tokens(32, 2, 1, 64, 64, act, F32, 9)
    x[1][:] = 2 * x[1][:1]
    check(x, DELTA)


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
def test_large_columns(act, rule):
    """Value channels of very different size."""
    x = tokens(64, 2, 1, 64, 64, act, F32, 10)
    x[2][..., 7] *= 2.0 ** 40
    x[2][..., 20] *= 2.0 ** -40
    check(x, rule)


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
def test_largest_finite_values(act, rule):
    """Values at the type's largest, forgotten with a gate of 0 and a beta of 0 before anything overflows."""
    x = tokens(64, 2, 1, 64, 64, act, F32, 11)
    x[2][50] = torch.finfo(act).max
    x[4][50] = 0.0
    clean = tuple(t.clone() for t in x)
    clean[2][50] = 0.0
    outs = []
    for y in (x, clean):
        o, out = torch.empty((64, 2, 64), dtype=act, device=DEV), torch.empty((1, 2, 64, 64), device=DEV)
        stepq.stepq_prompt(*(t.to(DEV) for t in y), o, out, rule, cu_seqlens=torch.tensor([0, 64], dtype=torch.int32, device=DEV))
        outs.append((o, out))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("rule", [DECAY, DELTA])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("j", [5, 40, 77])
def test_a_gate_below_zero(j, act, rule):
    """NaN from its token on in its head, and nothing else."""
    T = 130
    outs = []
    for a in (None, -0.5, -1e-30):
        x = tokens(T, 2, 1, 64, 64, act, F32, 12)
        if a is not None:
            x[3][j, 1] = a
        o, out = torch.empty((T, 2, 64), dtype=act, device=DEV), torch.empty((1, 2, 64, 64), device=DEV)
        stepq.stepq_prompt(*(t.to(DEV) for t in x), o, out, rule, cu_seqlens=torch.tensor([0, T], dtype=torch.int32, device=DEV))
        outs.append((o, out))
    (o, out), *rest = outs
    for po, pout in rest:
        assert torch.equal(po[:j], o[:j]) and torch.equal(po[:, 0], o[:, 0]) and torch.equal(pout[0, 0], out[0, 0])
        assert torch.isnan(po[j:, 1]).all() and torch.isnan(pout[0, 1]).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("how", ["random keys of norm 16", "equal keys of norm 8", "two keys of norm 2^70"])
def test_growth_past_fp32(how, act):
    """A state that passes fp32 inside a chunk does not reach the tokens before: those whose terms (of T's rows as of
    the outputs) are below 2^110 are what they are."""
    T = 64
    x = tokens(T, 2, 1, 64, 64, act, F32, 13)
    if how.startswith("two"):
        x[1][40:42] *= 2.0 ** 70
    else:
        x[1].mul_(16.0 if how.startswith("random") else 8.0)
        if how.startswith("equal"):
            x[1][:] = x[1][:1]
    S = torch.zeros(2, 64, 64)
    o, out = torch.empty((T, 2, 64), dtype=act, device=DEV), torch.empty((1, 2, 64, 64), device=DEV)
    stepq.stepq_prompt(*(t.to(DEV) for t in x), o, out, DELTA, cu_seqlens=torch.tensor([0, T], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    ro, _ = recurrence(*x, S, DELTA)
    mo, _ = magnitude(*x, S, DELTA)
    # T's rows, |M| |T| within them: what a token's u would be of values of size 1 everywhere
    rows, _ = magnitude(torch.ones_like(x[0]), x[1], torch.ones_like(x[2]), x[3], x[4], S, DELTA)
    safe = ((mo.amax((1, 2)) < 2.0 ** 110) & (rows.amax((1, 2)) < 2.0 ** 110)).tolist()
    n = safe.index(False) if False in safe else T
    assert 12 <= n < T                          # it does pass, and not at once
    off = (o[:n].cpu().double() - ro[:n]).abs()
    worst = (off / (3e-5 * mo[:n] + (0 if act == F32 else 2.0 ** -8) * ro[:n].abs())).amax((1, 2))
    assert (worst <= 1).all(), (n, worst)
    assert torch.isnan(o[T - 1]).all() and torch.isnan(out).all()
