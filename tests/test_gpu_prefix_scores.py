"""Scores with a large part in common: the softmax depends on their differences.

The scores are sums of 4096 (or its negative) and multiples of 1/8 below 8, exact in
fp32, so that the weights are off by the exponential's own rounding and the
scale's (2^-24 of a difference of 8): the bounds of test_gpu_prefix_weights.py for
bfloat16, 3e-5 of sum_t p_t |v_t| for float32.  A score rounded after the scale and
before the maximum is taken off would be wrong by 2^-12, and its weight with it.
lse is rounded five times on its way, by up to 2^-24 of itself each: the scale's
fp32 value, that times log2 e, the sum with log2 of the weights' sum, ln 2, and
the product with it."""
import pytest
import torch

from paper_2609_38169_amd import stepq
from test_gpu_prefix_product import reference
from test_gpu_prefix_weights import settled

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("scale", [1.0, 0.7, -0.7])
@pytest.mark.parametrize("offset", [4096.0, -4096.0])
@pytest.mark.parametrize("act,B,hq,hkv,D,P", [(F32, 3, 4, 2, 64, 90), (BF16, 3, 4, 2, 128, 90), (F32, 2, 2, 1, 256, 600),
                                              (BF16, 256, 16, 2, 64, 2333)])
def test_scores_with_a_common_part(act, B, hq, hkv, D, P, offset, scale):
    g = torch.Generator().manual_seed(1)
    page, own = 16, 20
    n_pre, n_own = -(-P // page), -(-own // page)
    n = n_pre + B * n_own
    q = torch.zeros((B, hq, D))
    q[..., 0], q[..., 1] = offset, 1.0
    k = torch.zeros((n, hkv, page, D))
    k[..., 0], k[..., 1] = 1.0, torch.randint(0, 64, (n, hkv, page), generator=g) / 8
    v = torch.randn((n, hkv, page, D), generator=g)
    i32 = lambda x: x.to(torch.int32).to(DEV)
    x = [q.to(act).to(DEV), k.to(act).to(DEV), v.to(act).to(DEV), i32(torch.arange(n_pre)), P,
         i32(n_pre + torch.arange(B * n_own)).view(B, n_own), i32(torch.randint(0, own + 1, (B,), generator=g))]
    o, lse = torch.empty((B, hq, D), dtype=act, device=DEV), torch.empty((B, hq), device=DEV)
    stepq.stepq_prefix_attention(*x, o, lse, scale)
    torch.cuda.synchronize()
    ro, size, rl = reference(*x, scale)
    if act == BF16:
        fine, by = settled(o, ro, size)
        assert fine, by
    else:
        off = (o.double() - ro).abs()
        assert (off <= 3e-5 * size).all(), float((off / size).max())
    assert ((lse.double() - rl).abs() <= 5 * 2.0 ** -24 * rl.abs()).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("act,B,hq,hkv,D,P", [(F32, 3, 4, 2, 64, 90), (BF16, 3, 4, 2, 128, 90), (BF16, 256, 16, 2, 64, 2333)])
def test_values_that_are_not_finite(act, B, hq, hkv, D, P, bad):
    """One of the prefix and one of a request's own: their columns of the rows that read them, and nothing else."""
    from test_gpu_prefix_product import inputs
    x = inputs(B, hq, hkv, D, P, own=5)
    x[:3] = [t.to(act) for t in x[:3]]
    x[6][:] = 3
    got = []
    for spoil in (False, True):
        if spoil:
            x[2][x[3][1].long(), 0, 3, 5] = bad
            x[2][x[5][1, 0].long(), hkv - 1, 2, 9] = bad
        o, lse = torch.empty((B, hq, D), dtype=act, device=DEV), torch.empty((B, hq), device=DEV)
        stepq.stepq_prefix_attention(*x, o, lse)
        got.append((o, lse))
    torch.cuda.synchronize()
    G = hq // hkv
    hit = torch.zeros((B, hq, D), dtype=torch.bool, device=DEV)
    hit[:, :G, 5] = True
    hit[1, hq - G:, 9] = True
    (clean, lse), (o, lse2) = got
    assert not torch.isfinite(o[hit]).any() and torch.equal(o[~hit], clean[~hit]) and torch.equal(lse, lse2)
