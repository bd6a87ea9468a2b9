"""Attention over a shared prefix: what a request gets does not depend on how
many others it comes with, beyond the output's own rounding.

Tolerance (bfloat16): the output is rounded once, by up to 2^-8 of its value
(8 significant bits).  Everything before that, the weights included, is kept to
16 bits or more: 2^-16 of sum_t p_t |v_t| for the weights' two planes, and 3e-5
of it for what is summed in 24 bits.  A weight rounded to 8 bits would be off by
up to 2^-8 of itself: sums over a few hundred keys then miss this bound wherever
the output is small beside sum_t p_t |v_t|."""
import pytest
import torch

from test_gpu_prefix_product import SHAPES, call, inputs, reference

pytestmark = pytest.mark.gpu


def settled(o, ro, size):
    off = (o.double() - ro).abs()
    bound = 2.0 ** -8 * ro.abs() + (2.0 ** -16 + 3e-5) * size
    return (off <= bound + 1e-30).all(), float(((off - bound) / size.clamp_min(1e-30)).max())


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("scale", [None, 0.02])
def test_weights_of_many_requests(shape, scale):
    """Softmax weights of the matrix-product form."""
    x = inputs(*shape)
    s = shape[3] ** -0.5 if scale is None else scale
    o, _ = call(x, s)
    ro, size, _ = reference(*x, s)
    fine, by = settled(o, ro, size)
    assert fine, by


def test_weights_of_few_requests():
    """The same bound on the form that takes few requests."""
    x = inputs(3, 16, 2, 64, 2333)
    o, _ = call(x, 0.125)
    ro, size, _ = reference(*x, 0.125)
    fine, by = settled(o, ro, size)
    assert fine, by
