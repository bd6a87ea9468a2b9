"""Limits of the calls on quantized caches at the C entry, and the largest sizes
that they take: host only, nothing here reaches a launch."""
import ctypes

import pytest
import torch

from paper_2609_38169_amd import stepq
from test_cache_host import UNSUPPORTED, P, attn, cache, size, tokens


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


@pytest.mark.parametrize("n_seq", [2 ** 31 - 64, 2 ** 31 - 1])
def test_sequences(n_seq):
    """The search for a token's sequence adds a 64th of them, and one, to an index: in 32 bits up to 2^31 - 65."""
    L, c, t = stepq.lib(), cache(), tokens(n_seq=n_seq)
    for f in (L.stepq_cache_write, L.stepq_cache_read):
        assert f(ctypes.byref(c), ctypes.byref(t), P, P, P, P, P, P, None) == UNSUPPORTED
        assert "sequences" in stepq.stepq_last_error()


def test_counts_that_no_field_holds():
    """The workspaces' sizes are of the counts asked for, or of none."""
    m = torch.zeros(4096, dtype=torch.uint8)
    m = m[-m.data_ptr() % 128:]
    c = stepq.Cache(1, 2, 1, 64, 8, memory=m)
    for f, args in ((stepq.stepq_cache_attention_workspace, (1, 2, 100, 0)),
                    (stepq.stepq_cache_select_workspace, (1, 2, 100, 5, 1, 1))):
        f(c, *args)
        for i in range(len(args)):
            for bad in (2 ** 32 + args[i], 2 ** 31, 0.5):
                with pytest.raises(ValueError):
                    f(c, *args[:i], bad, *args[i + 1:])
