"""Few query rows a key/value head over a long prefix, on both sides of where the
matrix-product form begins (33 rows at 256 dimensions, 65 otherwise): rows that
fill no tile, against the definition in 64 bits on the device.  Tolerances as in
test_gpu_prefix_weights.py."""
import math

import pytest
import torch

from test_gpu_prefix_product import call, inputs, reference
from test_gpu_prefix_weights import settled

pytestmark = pytest.mark.gpu

# (requests, query heads, key/value heads, head size, prefix)
SHAPES = [(1, 8, 8, 256, 33000), (1, 4, 1, 128, 70001), (17, 2, 2, 256, 33000), (32, 2, 2, 256, 33001), (33, 2, 2, 256, 33001),
          (64, 4, 4, 128, 20011), (65, 4, 4, 128, 20011), (17, 8, 2, 64, 70003)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_few_rows(shape):
    x = inputs(*shape, page=24, fill=math.nan)
    scale = shape[3] ** -0.5
    o, lse = call(x, scale)
    ro, size, rl = reference(*x, scale)
    fine, by = settled(o, ro, size)
    assert fine, by
    assert ((lse.double() - rl).abs() <= 3e-5 * rl.abs().clamp(min=1.0)).all()


@pytest.mark.parametrize("shape", [(33, 2, 2, 256, 33001), (65, 4, 4, 128, 20011)], ids=str)
def test_rows_without_a_key(shape):
    """Every page of the prefix missing, in a tile that is mostly empty."""
    x = inputs(*shape)
    x[3][:] = -1
    x[6][::2] = 0
    o, lse = call(x, 1.0)
    assert not o[::2].any() and (lse[::2] == -math.inf).all()
    ro, size, _ = reference(*x, 1.0)
    fine, by = settled(o, ro, size)
    assert fine, by
