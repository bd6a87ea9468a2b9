"""Limits of the calls on quantized caches at the C entry, and the largest sizes
that they take: host only, nothing here reaches a launch."""
import ctypes

import pytest

from paper_2609_38169_amd import stepq
from test_cache_host import UNSUPPORTED, P, attn, cache, size


@pytest.mark.parametrize("bits", [8, 4])
def test_scales(bits):
    """A scale times log2 e, and 16 of 4 bits, is finite."""
    L, c = stepq.lib(), cache(bits=bits)
    for scale in (2.0 ** 120, -2.0 ** 120, 2.0 ** -149, 0.0):
        assert size(L.stepq_cache_attention_workspace, c, attn(scale=scale))[0] == 0
    for scale in (2.0 ** 120 * (1 + 2.0 ** -23), -2.0 ** 121, 2.5e38, -3.4e38):
        d = attn(scale=scale)
        assert size(L.stepq_cache_attention_workspace, c, d)[0] == UNSUPPORTED and "scale" in stepq.stepq_last_error()
        assert L.stepq_cache_attention(ctypes.byref(c), ctypes.byref(d), P, P, P, P, None, P, P, P, 1 << 40, None) == UNSUPPORTED
