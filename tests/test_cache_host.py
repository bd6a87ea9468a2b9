"""What the calls on quantized caches refuse at the C entry, and their sizes:
host only, nothing here reaches a launch."""
import ctypes

import pytest
import torch

import _cache as C
from paper_2609_38169_amd import stepq

BAD, UNSUPPORTED = 1, 2
P = ctypes.c_void_p(4096)                # an aligned pointer that no refused call follows
ODD = ctypes.c_void_p(4097)


def make(kind, defaults, kw):
    defaults.update(kw)
    return kind(*defaults.values())


def cache(**kw):
    return make(stepq.stepq_cache_desc, dict(n_pages=8, n_kv_heads=2, page_size=16, head_dim=64, bits=8), kw)


def tokens(**kw):
    return make(stepq.stepq_cache_tokens, dict(n_tokens=10, n_seq=2, max_pages=3, act_dtype=stepq.STEPQ_BF16, k_stride=0,
                                               v_stride=0), kw)


def attn(**kw):
    return make(stepq.stepq_cache_attn_desc, dict(batch=2, n_q_heads=4, max_pages=100, act_dtype=stepq.STEPQ_BF16,
                                                  n_select=0, scale=1.0), kw)


def select(**kw):
    return make(stepq.stepq_cache_select_desc, dict(batch=2, n_q_heads=4, max_pages=100, act_dtype=stepq.STEPQ_BF16,
                                                    n_select=8, n_first=1, n_last=1), kw)


def size(f, *d):
    n = ctypes.c_size_t()
    return f(*(ctypes.byref(x) for x in d), ctypes.byref(n)), n.value


@pytest.mark.parametrize("bad,status", [
    (dict(n_pages=-1), BAD), (dict(n_kv_heads=0), BAD), (dict(page_size=0), BAD), (dict(head_dim=96), UNSUPPORTED),
    (dict(bits=16), UNSUPPORTED), (dict(bits=2), UNSUPPORTED), (dict(page_size=(1 << 20) + 1), UNSUPPORTED),
    (dict(n_pages=1 << 30), UNSUPPORTED),
])
def test_cache_descriptors(bad, status):
    """Every call on a cache refuses its descriptor."""
    L, c = stepq.lib(), cache(**bad)
    n = ctypes.c_size_t()
    b = ctypes.byref
    assert L.stepq_cache_bytes(b(c), b(n), None) == status and stepq.stepq_last_error()
    assert L.stepq_cache_write(b(c), b(tokens()), P, P, P, P, P, P, None) == status
    assert L.stepq_cache_read(b(c), b(tokens()), P, P, P, P, P, P, None) == status
    assert size(L.stepq_cache_attention_workspace, c, attn())[0] == status
    assert L.stepq_cache_attention(b(c), b(attn()), P, P, P, P, None, P, P, P, 1 << 40, None) == status
    assert L.stepq_cache_bounds(b(c), P, 2, 3, P, P, P, P, None) == status
    assert size(L.stepq_cache_select_workspace, c, select())[0] == status
    assert L.stepq_cache_select(b(c), b(select()), P, P, P, P, P, P, 1 << 40, None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(n_tokens=-1), BAD), (dict(n_seq=-1), BAD), (dict(max_pages=-1), BAD), (dict(act_dtype=2), BAD),
    (dict(k_stride=127), BAD), (dict(v_stride=-1), BAD), (dict(k_stride=(1 << 26) + 1), UNSUPPORTED),
    (dict(n_tokens=1 << 31), UNSUPPORTED), (dict(n_tokens=1 << 27), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED),
])
def test_token_descriptors(bad, status):
    L = stepq.lib()
    for f in (L.stepq_cache_write, L.stepq_cache_read):
        assert f(ctypes.byref(cache()), ctypes.byref(tokens(**bad)), P, P, P, P, P, P, None) == status
        assert stepq.stepq_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(n_q_heads=3), BAD), (dict(n_q_heads=0), BAD), (dict(batch=-1), BAD), (dict(max_pages=-1), BAD),
    (dict(act_dtype=7), BAD), (dict(n_select=-1), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD),
    (dict(max_pages=1 << 26), UNSUPPORTED), (dict(n_select=1 << 26), UNSUPPORTED), (dict(batch=1 << 22), UNSUPPORTED),
])
def test_attention_descriptors(bad, status):
    L = stepq.lib()
    assert size(L.stepq_cache_attention_workspace, cache(), attn(**bad))[0] == status
    assert stepq.stepq_last_error()
    assert L.stepq_cache_attention(ctypes.byref(cache()), ctypes.byref(attn(**bad)), P, P, P, P, P, P, P, P, 1 << 40,
                                   None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(n_q_heads=3), BAD), (dict(batch=-1), BAD), (dict(max_pages=-1), BAD), (dict(act_dtype=-1), BAD),
    (dict(n_select=0), BAD), (dict(n_first=-1), BAD), (dict(n_last=-1), BAD), (dict(n_first=5, n_last=4), BAD),
    (dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1), BAD), (dict(max_pages=1 << 26), UNSUPPORTED),
    (dict(batch=1 << 22), UNSUPPORTED), (dict(n_select=1 << 26), UNSUPPORTED),
])
def test_select_descriptors(bad, status):
    L = stepq.lib()
    assert size(L.stepq_cache_select_workspace, cache(), select(**bad))[0] == status
    assert stepq.stepq_last_error()
    assert L.stepq_cache_select(ctypes.byref(cache()), ctypes.byref(select(**bad)), P, P, P, P, P, P, 1 << 40, None) == status


def test_more_workgroups_than_a_launch_takes():
    L = stepq.lib()
    c = cache(n_kv_heads=64)
    many = dict(batch=1 << 17, n_q_heads=64)                 # 2^23 rows: one part each, or more
    assert size(L.stepq_cache_attention_workspace, c, attn(max_pages=16, **many)) == (0, 0)
    assert size(L.stepq_cache_attention_workspace, c, attn(max_pages=128, **many))[0] == UNSUPPORTED
    d = attn(max_pages=128, **many)
    assert L.stepq_cache_attention(ctypes.byref(c), ctypes.byref(d), P, P, P, P, None, P, P, P, 1 << 50, None) == UNSUPPORTED
    assert size(L.stepq_cache_select_workspace, c, select(max_pages=1024, **many))[0] == 0
    assert size(L.stepq_cache_select_workspace, c, select(max_pages=1025, **many))[0] == UNSUPPORTED


def refuse(call, args, changes):
    for i, x in changes:
        assert call(*(x if j == i else y for j, y in enumerate(args))) == BAD, (i, x)


def test_pointers_and_workspaces():
    L = stepq.lib()
    b = ctypes.byref
    n = ctypes.c_size_t()
    c, t, a, s = cache(), tokens(), attn(), select(max_pages=2000)
    assert L.stepq_cache_bytes(None, b(n), None) == BAD and L.stepq_cache_bytes(b(c), None, None) == BAD
    assert L.stepq_cache_attention_workspace(b(c), None, b(n)) == BAD
    assert L.stepq_cache_attention_workspace(b(c), b(a), None) == BAD
    assert L.stepq_cache_select_workspace(b(c), None, b(n)) == BAD
    assert L.stepq_cache_select_workspace(b(c), b(s), None) == BAD
    for f in (L.stepq_cache_write, L.stepq_cache_read):
        # desc, tokens, cache, table, starts, k, v are needed; without bounds every sequence has one token
        refuse(f, [b(c), b(t), P, P, P, P, P, P, None], [(i, None) for i in (0, 1, 2, 3, 4, 5, 6, 7)] +
               [(2, ctypes.c_void_p(4096 + 64)), (6, ODD), (7, ODD)])
        assert f(b(c), b(tokens(act_dtype=0)), P, P, P, P, ctypes.c_void_p(4098), P, None) == BAD
    need = size(L.stepq_cache_attention_workspace, c, a)[1]
    assert need > 0
    refuse(L.stepq_cache_attention, [b(c), b(a), P, P, P, P, None, P, None, P, need, None],
           [(i, None) for i in (0, 1, 2, 3, 4, 5, 7, 9)] + [(10, need - 1), (2, ODD), (3, ODD), (7, ODD), (9, ODD)])
    e = attn(n_select=3)                                     # a list of pages is needed then
    assert L.stepq_cache_attention(b(c), b(e), P, P, P, P, None, P, None, P, 1 << 40, None) == BAD
    refuse(L.stepq_cache_bounds, [b(c), P, 2, 3, P, P, P, P, None],
           [(i, None) for i in (0, 1, 4, 5, 6, 7)] + [(2, -1), (3, -1), (1, ODD), (7, ODD)])
    need = size(L.stepq_cache_select_workspace, c, s)[1]
    assert need > 0
    refuse(L.stepq_cache_select, [b(c), b(s), P, P, P, P, P, P, need, None],
           [(i, None) for i in (0, 1, 2, 3, 4, 5, 6, 7)] + [(8, need - 1), (2, ODD), (3, ODD), (7, ODD)])


def test_nothing_to_do():
    L = stepq.lib()
    b, c = ctypes.byref, cache()
    for f in (L.stepq_cache_write, L.stepq_cache_read):
        assert f(b(c), b(tokens(n_tokens=0, n_seq=0)), P, *[None] * 6) == 0
        assert f(b(c), b(tokens(n_tokens=0)), P, P, None, P, None, None, None) == 0
    assert L.stepq_cache_attention(b(c), b(attn(batch=0)), P, *[None] * 7, 0, None) == 0
    assert L.stepq_cache_bounds(b(c), P, 0, 3, *[None] * 5) == 0
    assert L.stepq_cache_bounds(b(c), P, 2, 0, *[None] * 5) == 0
    assert L.stepq_cache_select(b(c), b(select(batch=0)), *[None] * 6, 0, None) == 0
    assert size(L.stepq_cache_select_workspace, c, select(n_select=100))[1] == 0       # all pages are taken


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [1, 16, 24, 100])
def test_sizes(page, D, bits):
    n, r = stepq.stepq_cache_bytes(1000, 3, page, D, bits)
    assert r == C.record_bytes(page, D, bits) and n == 3000 * r
    most = (2 ** 37 - 1) // r                               # past 32 bits, up to 2^37 bytes
    assert stepq.stepq_cache_bytes(most, 1, page, D, bits)[0] == most * r
    with pytest.raises(stepq.StepqError):
        stepq.stepq_cache_bytes(most + 1, 1, page, D, bits)


def test_the_memory_stays():
    n = stepq.stepq_cache_bytes(2, 1, 4, 64, 8)[0]
    m = torch.zeros(n + 128, dtype=torch.uint8)
    m = m[-m.data_ptr() % 128:][:n]
    c = stepq.Cache(2, 1, 4, 64, 8, memory=m)
    assert c.memory is m and c.bytes == n
    with pytest.raises(AttributeError):
        c.memory = m.clone()
    with pytest.raises(ValueError):                          # not on a GPU
        c.write(*(torch.zeros(1, 1, 64),) * 2, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_values_that_no_field_holds():
    for bad in (2 ** 31, 0.5, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            stepq.stepq_cache_bytes(bad, 2, 16, 64, 8)
