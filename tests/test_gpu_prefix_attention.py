"""Attention over a shared prefix and each request's own pages, against its
definition in 64 bits.

Tolerances.  float32: scores and sums of at most a few thousand terms in fp32,
taken as 3e-5 of sum_t p_t |v_t| (the weights' relative error is the scores'
absolute one: |s| up to about 12 at 2^-24 each over D products).  bfloat16: the
weights and the output may each be rounded once to 8 bits: 2^-9 of
sum_t p_t |v_t| and of the output, and as much again for the 24-bit parts.
lse: 3e-5 of max(1, |lse|)."""
import math

import pytest
import torch

from paper_2609_38169_amd import stepq
from _sequence import attention

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def inputs(B, Hq, Hkv, D, prefix, lens, page, act, seed=1, spare=2, max_pages=None, fill=None):
    g = torch.Generator().manual_seed(seed)
    n_pre, n_own = -(-prefix // page), -(-max(lens, default=0) // page)
    n_own = n_own if max_pages is None else max_pages
    n = n_pre + B * n_own + spare
    rnd = lambda *s: torch.randn(s, generator=g).to(act)
    q, k, v = 2 * rnd(B, Hq, D), rnd(n, Hkv, page, D), rnd(n, Hkv, page, D)
    ids = torch.randperm(n, generator=g).to(torch.int32)
    pre, table = ids[:n_pre], ids[n_pre:n_pre + B * n_own].view(B, n_own).clone()
    lengths = torch.tensor(lens, dtype=torch.int32)
    if fill is not None:                       # what no request's tokens use
        used = torch.zeros((n, page), dtype=torch.bool)
        for t in range(prefix):
            used[pre[t // page], t % page] = True
        for b in range(B):
            for t in range(lens[b]):
                used[table[b, t // page], t % page] = True
        k.masked_fill_(~used[:, None, :, None], fill)
        v.masked_fill_(~used[:, None, :, None], fill)
        for b in range(B):
            table[b, -(-lens[b] // page):] = -7
    return q, k, v, pre, prefix, table, lengths


def call(x, scale=None, stream=None, lse=True, workspace=None):
    q, k, v, pre, prefix, table, lengths = (t.to(DEV) if isinstance(t, torch.Tensor) else t for t in x)
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    L = torch.full(q.shape[:2], 7.0, device=DEV) if lse else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    stepq.stepq_prefix_attention(q, k, v, pre, prefix, table, lengths, o, L, scale, workspace, stream)
    torch.cuda.synchronize()
    return o.cpu(), None if L is None else L.cpu()


def check(x, scale=None, **kw):
    o, lse = call(x, scale, **kw)
    ro, size, rl = attention(*x, x[0].shape[-1] ** -0.5 if scale is None else scale)
    off = (o.double() - ro).abs()
    bound = 3e-5 * size if o.dtype == F32 else 2.0 ** -8 * size + 2.0 ** -9 * ro.abs()
    assert (off <= bound + 1e-30).all(), ((off - bound) / (size + 1e-30)).max()
    if lse is not None:
        assert torch.equal(torch.isinf(lse), torch.isinf(rl))
        fine = ~torch.isinf(rl)
        assert ((lse.double() - rl).abs()[fine] <= 3e-5 * rl.abs().clamp(min=1.0)[fine]).all()
    return o, lse


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("prefix", [0, 1, 31, 64, 100, 1000])
@pytest.mark.parametrize("lens", [[1], [0, 1, 17, 64, 65], [300, 2, 0]], ids=lambda x: "-".join(map(str, x)))
def test_lengths(lens, prefix, act):
    check(inputs(len(lens), 8, 2, 128, prefix, lens, 16, act))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (5, 1), (16, 1), (20, 1), (40, 2)])
def test_heads(Hq, Hkv, D, act):
    check(inputs(3, Hq, Hkv, D, 130, [70, 1, 33], 16, act, seed=Hq))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("page", [1, 3, 24, 64, 100, 256])
def test_pages(page, act):
    check(inputs(3, 4, 2, 64, 333, [70, 101, 5], page, act, fill=math.nan))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf])
def test_what_is_not_used_does_not_matter(fill, act):
    """Pages and rows past a request's tokens hold anything, page ids past them too."""
    x = inputs(4, 4, 1, 128, 77, [0, 1, 50, 16], 16, act, fill=fill, max_pages=6)
    check(x)


@pytest.mark.parametrize("act", [F32, BF16])
def test_rows_without_a_key(act):
    x = inputs(3, 4, 2, 64, 0, [0, 5, 0], 16, act, max_pages=2)
    o, lse = check(x)
    assert not o[0].any() and not o[2].any() and torch.isinf(lse[0]).all() and (lse[0] < 0).all()


def test_no_pages_at_all():
    x = inputs(2, 4, 2, 64, 40, [0, 0], 16, BF16)
    assert x[5].shape == (2, 0)
    check(x)


@pytest.mark.parametrize("act", [F32, BF16])
def test_lowest_scores(act):
    """Keys whose scores are the type's lowest value or -inf: they get no weight beside others, and a row that
    has nothing else is empty at -inf."""
    x = inputs(2, 2, 1, 64, 20, [10, 3], 16, act)
    q, k, v, pre, prefix, table, lengths = x
    q[:, :, 0] = 1.0
    q[:, :, 1:] = 0.0
    low = torch.finfo(act).min
    k[pre[0].long(), 0, :16, 0] = low
    k[table[0, 0].long(), 0, 2:5, 0] = -math.inf
    check(x, scale=1.0)
    x2 = inputs(1, 2, 1, 64, 0, [10], 16, act)
    x2[0][:, :, 0], x2[0][:, :, 1:] = 1.0, 0.0
    x2[1][..., 0] = -math.inf
    o, lse = call(x2, scale=1.0)
    assert not o.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.1])
def test_scales(scale, act):
    """Scale 1 gives scores up to about 80: the running maximum carries them."""
    x = inputs(3, 4, 2, 64, 90, [40, 3, 65], 16, act)
    if scale == 1.0:
        x = (x[0] / 2,) + x[1:]
    o, lse = call(x, scale)
    ro, size, rl = attention(*x, scale)
    # the weights' error grows with the scores: |s| up to about 40 x 2^-22 of D = 64 fp32 terms
    tol = 2e-4 if act == F32 else 2.0 ** -7
    assert ((o.double() - ro).abs() <= tol * size).all()
    assert ((lse.double() - rl).abs() <= 3e-5 * rl.abs().clamp(min=1.0)).all()


def test_a_value_that_is_not_finite_stays_in_its_column():
    """A used value that is not finite reaches its own column of the requests that read it."""
    x = inputs(3, 2, 1, 64, 40, [20, 20, 20], 16, BF16)
    clean, _ = call(x)
    x[2][x[5][1, 0].long(), 0, 3, 9] = math.nan
    o, _ = call(x)
    hit = torch.zeros(o.shape, dtype=torch.bool)
    hit[1, :, 9] = True
    assert torch.isnan(o[hit]).all() and torch.equal(o[~hit], clean[~hit])


@pytest.mark.parametrize("act", [F32, BF16])
def test_page_ids_out_of_range_are_left_out(act):
    x = inputs(2, 4, 2, 64, 70, [50, 20], 16, act)
    x[3][2], x[5][0, 1] = -1, 10 ** 6
    check(x)


def test_lengths_past_the_pages_are_cut():
    x = inputs(2, 4, 2, 64, 10, [32, 5], 16, BF16)
    x[6][0] = 4000
    check(x)


@pytest.mark.parametrize("act", [F32, BF16])
def test_many_requests(act):
    check(inputs(70, 4, 1, 64, 257, [(13 * i) % 41 for i in range(70)], 16, act))


@pytest.mark.parametrize("act", [F32, BF16])
def test_long(act):
    check(inputs(2, 4, 2, 64, 9000, [5000, 3], 64, act))


def test_stream_and_no_lse():
    x = inputs(3, 4, 2, 64, 90, [40, 3, 65], 16, BF16)
    a, _ = call(x)
    b, none = call(x, stream=torch.cuda.Stream(), lse=False)
    assert none is None and torch.equal(a, b)


def test_own_workspace():
    x = inputs(3, 4, 2, 64, 90, [40, 3, 65], 16, BF16)
    n = stepq.stepq_prefix_attention_workspace(3, 4, 2, 64, 90, x[5].shape[1], 16)
    a, _ = call(x)
    b, _ = call(x, workspace=torch.full((max(n, 1),), 255, dtype=torch.uint8, device=DEV))
    assert torch.equal(a, b)


def test_graph():
    """A decode loop's replay: lengths grow and queries change in the captured buffers."""
    q, k, v, pre, prefix, table, lengths = (t.to(DEV) if isinstance(t, torch.Tensor) else t
                                            for t in inputs(4, 8, 2, 128, 200, [5, 60, 1, 31], 16, BF16, max_pages=8))
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    run = lambda: stepq.stepq_prefix_attention(q, k, v, pre, prefix, table, lengths, o, lse)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        q.copy_(torch.randn_like(q))
        lengths += 9
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        o.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse)


def test_offsets_over_32_bits():
    """Pages beyond 2^32 elements of the cache."""
    n, page, D = 8200, 64, 256                      # 8200 x 32 x 64 x 256 elements, 2^32 at page 8192
    Hkv = 32
    k, v = (torch.empty((n, Hkv, page, D), dtype=BF16, device=DEV) for _ in range(2))
    ids = [8199, 0, 8195, 8193]
    small = inputs(2, Hkv, Hkv, D, 70, [100, 20], page, BF16)
    ks, vs = torch.zeros(4, Hkv, page, D, dtype=BF16), torch.zeros(4, Hkv, page, D, dtype=BF16)
    g = torch.Generator().manual_seed(3)
    ks.copy_(torch.randn(ks.shape, generator=g)), vs.copy_(torch.randn(ks.shape, generator=g))
    for i, p in enumerate(ids):
        k[p], v[p] = ks[i].to(DEV), vs[i].to(DEV)
    q, lengths = small[0], torch.tensor([100, 20], dtype=torch.int32)
    table = torch.tensor([[2, 3], [1, 0]], dtype=torch.int32)
    pre = torch.tensor([0, 1], dtype=torch.int32)
    back = torch.tensor(ids, dtype=torch.int32)
    o = torch.empty(q.shape, dtype=BF16, device=DEV)
    stepq.stepq_prefix_attention(q.to(DEV), k, v, back[pre.long()].to(DEV), 70, back[table.long()].to(DEV),
                                 lengths.to(DEV), o)
    torch.cuda.synchronize()
    ro, size, _ = attention(q, ks, vs, pre, 70, table, lengths, D ** -0.5)
    assert ((o.cpu().double() - ro).abs() <= 2.0 ** -8 * size + 2.0 ** -9 * ro.abs()).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("B", [2, 40])
def test_caches_without_a_page(act, B):
    """No page at all, yet page ids and lengths that ask for some: every row is empty."""
    x = list(inputs(B, 4, 2, 64, 40, [9] * B, 16, act))
    x[1], x[2] = x[1][:0], x[2][:0]
    o, lse = call(tuple(x))
    assert not o.any() and (lse == -math.inf).all()


def test_refusals():
    q, k, v, pre, prefix, table, lengths = (t.to(DEV) if isinstance(t, torch.Tensor) else t
                                            for t in inputs(2, 4, 2, 64, 40, [5, 6], 16, BF16))
    o = torch.empty_like(q)
    f = stepq.stepq_prefix_attention
    with pytest.raises(TypeError):
        f(q.half(), k, v, pre, prefix, table, lengths, o)
    with pytest.raises(TypeError):
        f(q, k.float(), v, pre, prefix, table, lengths, o)
    with pytest.raises(ValueError):
        f(q, k, v[:-1], pre, prefix, table, lengths, o)
    with pytest.raises(ValueError):
        f(q, k, v, pre[:1], prefix, table, lengths, o)
    with pytest.raises(ValueError):
        f(q, k, v, None, prefix, table, lengths, o)
    with pytest.raises(ValueError):
        f(q, k, v, pre, -1, table, lengths, o)
    with pytest.raises(TypeError):
        f(q, k, v, pre, prefix, table.long(), lengths, o)
    with pytest.raises(ValueError):
        f(q, k, v, pre, prefix, table, lengths[:1], o)
    with pytest.raises(ValueError):
        f(q.transpose(0, 1), k, v, pre, prefix, table, lengths, o)
    with pytest.raises(stepq.StepqError):
        f(q, k, v, pre, prefix, table, lengths, o, scale=math.inf)
    with pytest.raises(stepq.StepqError):
        f(q[..., :32].contiguous(), k[..., :32].contiguous(), v[..., :32].contiguous(), pre, prefix, table, lengths,
          o[..., :32].contiguous())
    with pytest.raises(stepq.StepqError):
        f(q[:, :3].contiguous(), k, v, pre, prefix, table, lengths, o[:, :3].contiguous())
    with pytest.raises((ValueError, TypeError)):
        f(q, k, v, pre, prefix, table, lengths, o, workspace=torch.empty(4, device=DEV))


@pytest.mark.parametrize("act", [F32, BF16])
def test_binding_paths_agree(act, monkeypatch):
    """The native argument path and the Python one make the same calls."""
    x = inputs(3, 4, 2, 128, 90, [40, 3, 65], 16, act)
    a, b = call(x), call(x, scale=0.25)
    monkeypatch.setattr(stepq, "_native", stepq._PythonChecks)
    c, d = call(x), call(x, scale=0.25)
    assert all(torch.equal(p, q) for p, q in zip(a + b, c + d))
