"""Attention over quantized caches at the ends of the numbers' range: keys and
values up to the type's largest, sums close to it, and queries of single
dimensions many times the others.

Tolerances, from the arithmetic.  Products of queries (8 bits, or planes of 24) and
codes (7 bits) are exact.  A score is a sum of D of them, a product with each
group's scale and a place in the exponent: D + 8 roundings of at most 2^-23 (the
matrix cores need not round to the nearest) of sum_d |q_d k_d|, together e; an
exponential is off by 2^-23 more.  Weights are so off by 2 e + 2^-22, their planes
by 2^-16 (bfloat16) or 2^-22 (float32), and the two sums of n terms by n 2^-23 each,
all relative; the output is rounded once, by half a step.  lse is off by e and the
sum's n 2^-23, and by 2^-22 of itself."""
import math

import pytest
import torch

import _cache as C
from test_gpu_cache_attention import Case

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
LARGEST = 2.0 ** 128 * (1 - 2.0 ** -24)


def set_scales(c, which, s):
    """Scales s [n_pages][Hkv][P] (bfloat16 values) of all groups of the keys (0) or values (1) that are, codes as they are."""
    part = C.parts(c.mem, c.P, c.D, c.bits)[2 + which].view(torch.bfloat16)
    held, each = (c.K, c.V)[which], c.D // part.shape[-1]
    there = torch.isfinite(part)
    old = torch.where(there, part.double(), 1.0)
    s = s.to(torch.bfloat16)[..., None].expand(part.shape)
    held.mul_((s.double() / old).repeat_interleave(each, -1))
    held.copy_(torch.round(held / s.double().repeat_interleave(each, -1)) * s.double().repeat_interleave(each, -1))
    part.copy_(torch.where(there, s, part))


def check(c, scale):
    o, lse = c.call(scale)
    ro, size, rl = C.attention(c.q, c.K, c.V, c.table, c.lengths, None, scale)
    B, Hq, D = c.q.shape
    G = Hq // c.Hkv
    for b in range(B):
        n = int(c.lengths[b])
        k = c.K[c.table[b].long()].transpose(1, 2).reshape(-1, c.Hkv, D)[:n]                # [n][Hkv][D]
        for h in range(Hq):
            terms = (c.q[b, h].double().abs() * k[:, h // G].abs()).sum(-1).max() * abs(scale)
            e = (D + 8) * 2.0 ** -23 * float(terms)
            w = 2 * e + 2.0 ** -22 + (2.0 ** -16 if o.dtype == BF16 else 2.0 ** -22) + 2 * n * 2.0 ** -23
            off = (o[b, h].double() - ro[b, h]).abs()
            bound = w * size[b, h] + (2.0 ** -8 if o.dtype == BF16 else 2.0 ** -24) * ro[b, h].abs()
            assert (off <= bound).all(), (b, h, float((off / size[b, h]).max()), w)
            gap = abs(float(lse[b, h]) - float(rl[b, h]))
            assert gap <= e + n * 2.0 ** -23 + 2.0 ** -22 * (1 + abs(float(rl[b, h]))), (b, h, gap, e)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_up_to_the_largest(D, bits, act):
    """Rows of up to 2.9e38 (4 bits) and 3.2e38, with queries that bring the scores to a few units."""
    c = Case([70, 1, 33, 1300], 4, 2, D, 16, bits, act, seed=D)
    set_scales(c, 0, torch.full(c.K.shape[:3], 1.9375 * 2.0 ** (124 if bits == 4 else 120)))
    assert 2.8e38 < c.K.abs().max() < 3.3e38
    c.q = (c.q.float() * 2.0 ** -60).to(act)
    check(c, 2.0 ** -66 * D ** -0.5)


def largest_scale(n, bits):
    """The largest scale of values of which n stay in the range: n times the largest magnitude (a sixteenth of it of 4
    bits) below the type's largest, and that itself at most 3.3e38."""
    top = C.TOP[bits]
    s = torch.tensor(min(3.3e38 / top, LARGEST / n / top * (16 if bits == 4 else 1)), dtype=torch.float32)
    return (s.view(torch.int32) & -65536).view(torch.float32)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n", [1, 2, 16, 100, 700, 5000])
def test_values_up_to_the_largest(n, bits, act):
    c = Case([n], 4, 2, 64, 16, bits, act, seed=n)
    set_scales(c, 1, largest_scale(n, bits).expand(c.V.shape[:3]))
    check(c, 64 ** -0.5)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n", [300, 700, 3000])
def test_sums_of_scores_that_rise(n, bits, act):
    """Scores that rise by a factor of 45 (less than 2^6) after the first tiles, values of one sign at the largest: sums of
    weights above 1 would pass the range."""
    D = 64
    c = Case([n], 2, 1, D, 16, bits, act, seed=n)
    pos = torch.zeros(c.K.shape[:3], dtype=torch.int64)
    for t in range(n):
        pos[c.table[0, t // 16], 0, t % 16] = t % 1024 if n > 768 else t
    for i, x in ((0, c.K), (1, c.V)):                # every key is the same row but for its scale, every value all top codes
        codes = torch.full((D,), C.TOP[bits], dtype=torch.float64)
        C.parts(c.mem, 16, D, bits)[i][:] = C.rows_to_bytes(codes, bits)
        part = C.parts(c.mem, 16, D, bits)[2 + i].view(torch.bfloat16)
        part.copy_(torch.where(torch.isfinite(part), torch.ones_like(part), part))
        x.copy_(codes.expand(x.shape))
    set_scales(c, 0, torch.where(pos < 128, 1.0, 1.5).float())
    set_scales(c, 1, largest_scale(n, bits).expand(c.V.shape[:3]))
    c.q = torch.ones_like(c.q)
    check(c, math.log(45.0) / (0.5 * D * C.TOP[bits]))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("big", [10, 14, 18])
def test_queries_with_a_large_dimension(big, bits, D, act):
    """One query dimension of 2^big where every key's code is 0 adds nothing to the scores, nor to their error."""
    c = Case([70, 1, 33, 1300], 8, 2, D, 16, bits, act, seed=D + big)
    dims = [3, D // 2 + 5, D - 1]
    for d in dims:
        part = C.parts(c.mem, c.P, D, bits)[0]
        if bits == 8:
            part[..., d] = 0
        else:
            w, j = d % (D // 4), d // (D // 4)
            part[..., 2 * w + j // 2] &= 0xf0 if j % 2 == 0 else 0x0f
        c.K[..., d] = 0.0
    g = torch.Generator().manual_seed(big)
    q = c.q.float()
    for d in dims:
        q[..., d] = 2.0 ** big * (1 + torch.rand(q.shape[:2], generator=g)) * (1 if d == dims[0] else -0.3)
    c.q = q.to(act)
    check(c, D ** -0.5)
