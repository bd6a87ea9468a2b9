"""The bounds of a quantized cache's pages and the pages that a query selects by
them, against their definitions.

Tolerance: none.  Bounds are held values rounded one way; scores are sums in 64
bits rounded once, so that whatever the order of summation the same pages have
the highest ones, ties going to the lowest position."""
import math

import pytest
import torch

import _cache as C
from paper_2609_38169_amd import stepq

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def cache_of(mem, P, D, bits):
    return stepq.Cache(mem.shape[0], mem.shape[1], P, D, bits, memory=mem.to(DEV).flatten())


def same(a, b):
    """Equal as bfloat16 values, NaN to NaN."""
    return torch.equal(torch.nan_to_num(a.float().cpu(), nan=12345.0), torch.nan_to_num(b.float().cpu(), nan=12345.0))


def check_bounds(mem, K, table, starts, lengths, P, D, bits):
    n_pages, Hkv = mem.shape[:2]
    g = torch.Generator().manual_seed(9)
    want = torch.randn((n_pages, Hkv, 2, D), generator=g).to(BF16)
    got = want.to(DEV)
    cache_of(mem, P, D, bits).bounds(table.to(DEV), starts.to(DEV), lengths.to(DEV), got)
    for b in range(table.shape[0]):
        n = min(max(int(lengths[b]), 0), table.shape[1] * P)
        if int(starts[b]) < 0 or int(starts[b]) >= n:
            continue
        for p in range(int(starts[b]) // P, (n - 1) // P + 1):
            page = int(table[b, p])
            if 0 <= page < n_pages:
                for h in range(Hkv):
                    want[page, h] = C.bounds_of(K[page, h, :min(P, n - p * P)])
    assert same(got, want)
    return got.cpu()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (256, 16), (64, 1), (128, 24), (64, 100), (128, 256)])
def test_bounds(D, P, bits):
    lens, starts = [100, 37, 0, 260, 5, 64], [0, 36, 0, 130, 5, 1000]
    M = -(-260 // P)
    mem, K, V = C.fill(len(lens) * M + 2, 2, P, D, bits, seed=P)
    g = torch.Generator().manual_seed(P)
    table = torch.randperm(mem.shape[0], generator=g).to(torch.int32)[:len(lens) * M].view(-1, M)
    table[3, M - 1] = -1 if P > 100 else mem.shape[0]
    check_bounds(mem, K, table, torch.tensor(starts, dtype=torch.int32), torch.tensor(lens, dtype=torch.int32), P, D, bits)


@pytest.mark.parametrize("bits", [8, 4])
def test_bounds_of_keys_that_are_not_finite(bits):
    """NaN in its group of dimensions, and no farther; rows past the length do not count."""
    mem, K, V = C.fill(4, 2, 16, 128, bits, seed=3)
    s = C.parts(mem, 16, 128, bits)[2].view(torch.int16)
    s[1, 0, 4, 0] = 0x7fc0
    K[1, 0, 4, :64 if bits == 4 else 128] = math.nan
    s[2, :, 9:] = 0x7fc0
    table = torch.tensor([[0, 1], [3, 2]], dtype=torch.int32)
    got = check_bounds(mem, K, table, torch.tensor([0, 20], dtype=torch.int32), torch.tensor([32, 25], dtype=torch.int32), 16,
                       128, bits)
    assert torch.isnan(got[1, 0, :, 3]).all() and not torch.isnan(got[2]).any()


def test_bounds_of_many_pages():
    """More pages than workgroups take at once."""
    P, D = 1, 64
    mem, K, V = C.fill(9000, 1, P, D, 8, seed=1)
    table = torch.randperm(9000).to(torch.int32)[None]
    check_bounds(mem, K, table, torch.tensor([17], dtype=torch.int32), torch.tensor([8999], dtype=torch.int32), P, D, 8)


def check_select(q, bounds, table, lengths, P, S, first, last, bits=8, workspace=False, stream=None):
    n_pages, Hkv, _, D = bounds.shape
    cache = stepq.Cache(n_pages, Hkv, P, D, bits)
    got = torch.full((table.shape[0], Hkv, S), 77, dtype=torch.int32, device=DEV)
    ws = None
    if workspace:
        n = stepq.stepq_cache_select_workspace(cache, table.shape[0], q.shape[1], table.shape[1], S, first, last, q.dtype)
        ws = torch.full((max(n, 1),), 255, dtype=torch.uint8, device=DEV)
    args = [x.to(DEV) for x in (q, bounds, table, lengths)]
    torch.cuda.synchronize()
    cache.select(*args, got, first, last, ws, stream)
    torch.cuda.synchronize()
    want = C.select(q, bounds, table, lengths, P, S, first, last)
    assert torch.equal(got.cpu(), want)
    return want


# columns of the page table that lead to each form of the selection (up to 1024, more): as many as the pages, or more,
# which no request uses
FORMS = [None, 1500]


def setup(lens, Hq, Hkv, D, P, act, seed=1, max_pages=None):
    g = torch.Generator().manual_seed(seed)
    B, M = len(lens), -(-max(lens) // P) if max_pages is None else max_pages
    n = B * M + 2
    lo, hi = torch.randn((2, n, Hkv, D), generator=g).sort(0).values
    bounds = torch.stack([lo, hi], 2).to(BF16)
    table = torch.randperm(n, generator=g).to(torch.int32)[:B * M].view(B, M)
    return (torch.randn((B, Hq, D), generator=g).to(act), bounds, table, torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("M", FORMS)
def test_select(M, D, act):
    for Hq, Hkv in ((1, 1), (6, 2), (20, 1)):
        x = setup([100, 0, 1, 700, 333, 161], Hq, Hkv, D, 16, act, seed=D, max_pages=M)
        for S, first, last in ((10, 1, 1), (1, 0, 0), (1, 0, 1), (7, 3, 4), (12, 0, 2), (100, 1, 1)):
            check_select(*x, 16, S, first, last)


@pytest.mark.parametrize("pages", [255, 1023, 1024, 1025, 8192, 8200])
def test_pages_at_the_borders_of_the_forms(pages):
    x = setup([pages, pages - 1, pages - 3, 30], 2, 1, 64, 1, BF16, max_pages=pages)
    for S, first, last in ((20, 1, 2), (pages - 1, 0, 1), (pages // 2, 0, 0)):
        check_select(*x, 1, S, first, last)


@pytest.mark.parametrize("P", [1, 24, 64])
def test_pages_and_workspace(P):
    x = setup([1000, 64, 65], 4, 2, 64, P, BF16)
    check_select(*x, P, 5, 1, 2, workspace=True)
    check_select(*x, P, 5, 1, 2, stream=torch.cuda.Stream())


def test_long():
    """More pages than one pass over a request's scores holds."""
    x = setup([20000, 12345], 4, 1, 64, 1, BF16)
    check_select(*x, 1, 3000, 4, 8)
    check_select(*x, 1, 1, 0, 0)


@pytest.mark.parametrize("M", FORMS)
def test_equal_scores_go_to_the_lowest_position(M):
    q, bounds, table, lengths = setup([1600, 1599], 2, 1, 64, 4, F32, max_pages=M)
    bounds[:] = bounds[0]
    want = check_select(q, bounds, table, lengths, 4, 30, 2, 3)
    assert want[0, 0].tolist() == list(range(27)) + [397, 398, 399]
    bounds[1::2] *= 0.5                                # two values, one of them many times
    check_select(q, bounds, table, lengths, 4, 333, 2, 3)


@pytest.mark.parametrize("M", FORMS)
def test_scores_that_differ_in_their_last_place(M):
    """Neighbouring scores, some equal once rounded: whole multiples of 2^-30 beside 1."""
    q, bounds, table, lengths = setup([800], 1, 1, 64, 4, F32, max_pages=M)
    q[:] = 0.0
    q[0, 0, 0], q[0, 0, 1] = 1.0, 2.0 ** -30
    bounds[:] = 0.0
    bounds[:, 0, 1, 0] = 1.0
    g = torch.Generator().manual_seed(1)
    bounds[:, 0, 1, 1] = torch.randint(0, 200, (bounds.shape[0],), generator=g).to(BF16)
    check_select(q, bounds, table, lengths, 4, 50, 0, 1)


@pytest.mark.parametrize("M", FORMS)
def test_scores_that_are_not_finite(M):
    """NaN counts as the highest, then +inf; -inf as the lowest but for pages that are none."""
    q, bounds, table, lengths = setup([400, 400], 2, 1, 64, 4, F32, max_pages=M)
    q[:, :, 0] = 1.0
    n = [int(x) for x in table[0]]
    for i, x in ((10, math.nan), (40, math.nan), (20, math.inf), (60, math.inf)):
        bounds[n[i], 0, 1, 0] = x
    q[:, :, 1] = -1.0
    for i in (30, 31, 32):
        bounds[n[i], 0, 0, 1] = math.inf               # -1 x inf
    table[0, 50], table[0, 51] = -1, bounds.shape[0]
    for S in (4, 6, 8, 96, 98):
        check_select(q, bounds, table, lengths, 4, S, 0, 1)


@pytest.mark.parametrize("M", [40, 1500])
def test_what_is_not_used_does_not_matter(M):
    """Page ids past a request's pages, and the bounds of pages that always are taken."""
    q, bounds, table, lengths = setup([100, 90], 4, 2, 64, 4, BF16, max_pages=M)
    for b in range(2):
        pages = -(-int(lengths[b]) // 4)
        table[b, pages:] = -5
        bounds[table[b, [0, pages - 1, pages - 2]].long()] = math.nan
    check_select(q, bounds, table, lengths, 4, 9, 1, 2)


@pytest.mark.parametrize("M", FORMS)
def test_queries_of_any_size(M):
    """Sums over the heads and dimensions in 64 bits: queries of very different sizes, and zeros."""
    q, bounds, table, lengths = setup([400], 16, 1, 128, 4, F32, max_pages=M)
    q *= 2.0 ** torch.randint(-30, 30, q.shape, generator=torch.Generator().manual_seed(1))
    check_select(q, bounds, table, lengths, 4, 20, 1, 1)
    check_select(torch.zeros_like(q), bounds, table, lengths, 4, 20, 1, 1)


@pytest.mark.parametrize("M", FORMS)
def test_a_request_of_no_pages(M):
    q, bounds, table, lengths = setup([0, 0], 2, 1, 64, 4, BF16, max_pages=M)
    want = check_select(q, bounds, table, lengths, 4, 3, 1, 1)
    assert (want == -1).all()


def test_refusals():
    q, bounds, table, lengths = (x.to(DEV) for x in setup([100, 90], 4, 2, 64, 4, BF16))
    cache = stepq.Cache(bounds.shape[0], 2, 4, 64, 8)
    sel = torch.zeros((2, 2, 6), dtype=torch.int32, device=DEV)
    f = cache.select
    with pytest.raises(TypeError):
        f(q.half(), bounds, table, lengths, sel)
    with pytest.raises(TypeError):
        f(q, bounds.float(), table, lengths, sel)
    with pytest.raises(ValueError):
        f(q, bounds[:-1], table, lengths, sel)
    with pytest.raises(ValueError):
        f(q, bounds, table, lengths, sel[:, :1])
    with pytest.raises(ValueError):
        f(q, bounds, table, lengths, sel[:, :, :0])
    with pytest.raises(TypeError):
        f(q, bounds, table, lengths, sel.long())
    with pytest.raises(stepq.StepqError):
        f(q, bounds, table, lengths, sel, 4, 3)
    with pytest.raises(stepq.StepqError):
        f(q, bounds, table, lengths, sel, -1, 3)
    with pytest.raises(ValueError):
        f(q, bounds, table, lengths, sel, 0.5, 3)
    with pytest.raises(stepq.StepqError):
        f(q[:, :3].contiguous(), bounds, table, lengths, sel)
    with pytest.raises(ValueError):
        cache.bounds(table, lengths[:1], lengths, bounds)
    with pytest.raises(TypeError):
        cache.bounds(table, lengths, lengths, bounds.float())
    with pytest.raises(ValueError):
        cache.bounds(table, lengths, lengths, bounds[:1])
