"""Calls on quantized caches that are large enough for what small ones do not
reach: workgroups that take several rows or page groups in turn, ranges of more
than 256 tokens or pages, selected pages over several ranges; and bounds of
sequences that are wrong, inside memory whose surroundings are watched.

Tolerances: those of test_gpu_cache_attention.py for attention, none for what is
held and selected."""
import pytest
import torch

import _cache as C
from paper_2609_38169_amd import stepq
from test_gpu_cache_attention import Case
from test_gpu_cache_select import check_select, setup

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


# ---------------------------------------------------------------------------
# rows

@pytest.mark.parametrize("T,Hkv,D,bits,act", [(40001, 5, 128, 8, BF16), (40001, 5, 128, 4, F32), (41003, 3, 256, 4, BF16),
                                              (90007, 3, 64, 8, F32)])
def test_workgroups_of_several_rows(T, Hkv, D, bits, act):
    """A workgroup takes 4096 / D tokens to write, 2048 / D to read; from 8192 and 2048 workgroups on they take several of a
    token's 2 Hkv rows, in steps that do not divide them."""
    P, n = 24, 7
    g = torch.Generator().manual_seed(D + bits)
    lens = [T // n + i - 3 for i in range(n - 1)]
    lens.append(T - sum(lens))
    starts = [0, 5, 23, 24, 100, 7, 1]
    M = max(-(-(l + s) // P) for l, s in zip(lens, starts))
    n_pages = n * M + 2
    k, v = (torch.randn((T, Hkv, D), generator=g).to(act) for _ in range(2))
    table = torch.randperm(n_pages, generator=g).to(torch.int32)[:n * M].view(n, M)
    mem = torch.randint(0, 256, (n_pages, Hkv, C.record_bytes(P, D, bits)), generator=g, dtype=torch.uint8)
    cache = stepq.Cache(n_pages, Hkv, P, D, bits, memory=mem.to(DEV).flatten())
    cu = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0, dtype=torch.int32)
    at = [x.to(DEV) for x in (table, torch.tensor(starts, dtype=torch.int32))]
    cache.write(k.to(DEV), v.to(DEV), *at, cu.to(DEV))
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(lens))
    pos = torch.arange(T) - cu[seq] + torch.tensor(starts)[seq]
    page, row = table[seq, pos // P].long(), pos % P
    want = []
    for i, x in ((0, k), (1, v)):
        c, s = C.quantize(x, bits)
        C.parts(mem, P, D, bits)[i][page, :, row] = C.rows_to_bytes(c, bits)
        C.parts(mem, P, D, bits)[2 + i][page, :, row] = C.scales_to_bytes(s)
        want.append(C.value(c, s).to(act))
    assert torch.equal(cache.memory.cpu().view(mem.shape), mem)
    got = [torch.full((T, Hkv, D), 7.0, dtype=act, device=DEV) for _ in range(2)]
    cache.read(*at, *got, cu.to(DEV))
    for x, y in zip(got, want):
        assert torch.equal(x.cpu(), y)


@pytest.mark.parametrize("bits", [8, 4])
def test_wrong_bounds_touch_nothing_else(bits):
    """Bounds that go down or lie outside the tokens: the memory around the cache and around what is read, and the pages
    that no table names, stay as they are; what is read of a token is what the cache holds of it, zero, or untouched."""
    Hkv, P, D, n, T, edge = 1, 4, 64, 3, 18, 4096
    g = torch.Generator().manual_seed(bits)
    k, v = (torch.randn((T, Hkv, D), generator=g).to(BF16) for _ in range(2))
    table = torch.tensor([[1, 6], [9, 4], [3, 12]], dtype=torch.int32)
    n_pages, starts = 14, torch.tensor([0, 2, 1], dtype=torch.int32)
    size, rec = stepq.stepq_cache_bytes(n_pages, Hkv, P, D, bits)
    for bad in ([0, 12, 3, 18], [5, -4, 100, 7], [-2 ** 31, 0, 2 ** 31 - 1, 4], [18, 12, 6, 0], [0, 0, 2 ** 31 - 1, 2 ** 31 - 1],
                [-7, -7, -7, 18]):
        whole = torch.randint(0, 256, (size + 2 * edge,), generator=g, dtype=torch.uint8)
        whole[edge:edge + size] = 0
        mine = whole.to(DEV)
        cache = stepq.Cache(n_pages, Hkv, P, D, bits, memory=mine[edge:edge + size])
        cu = torch.tensor(bad, dtype=torch.int32, device=DEV)
        cache.write(k.to(DEV), v.to(DEV), table.to(DEV), starts.to(DEV), cu)
        after = mine.cpu()
        assert torch.equal(after[:edge], whole[:edge]) and torch.equal(after[edge + size:], whole[edge + size:])
        pages = after[edge:edge + size].view(n_pages, rec)
        others = [p for p in range(n_pages) if p not in table.flatten().tolist()]
        assert not pages[others].any()
        wide = torch.full((2, 3 * T, Hkv, D), 7.0, dtype=BF16, device=DEV)
        cache.read(table.to(DEV), starts.to(DEV), wide[0, T:2 * T], wide[1, T:2 * T], cu)
        assert torch.equal(mine.cpu(), after)
        got = wide.cpu().float()
        assert (got[:, :T] == 7.0).all() and (got[:, 2 * T:] == 7.0).all()
        got = got[:, T:2 * T].reshape(2, T, D)
        for x, y in zip(got, (k, v)):
            held = C.held(y[:, 0], bits).to(BF16).float()
            for t in range(T):
                known = (x[t] == 7.0).all() or not x[t].any() or torch.equal(x[t], held[t])
                assert known, (bad, t)


# ---------------------------------------------------------------------------
# selection

@pytest.mark.parametrize("D,M", [(64, 700), (128, 300), (256, 150)])
@pytest.mark.parametrize("act", [F32, BF16])
def test_scores_of_page_groups_in_turn(act, D, M):
    """512 (request, head) pairs leave 4 workgroups each, which take groups of 4096 / D pages in turn; requests end inside
    any of them."""
    P, B, Hkv = 2, 64, 8
    lens = [max(0, M * P - 37 * i) for i in range(B)]
    x = setup(lens, 2 * Hkv, Hkv, D, P, act, seed=D, max_pages=M)
    for S, first, last in ((20, 1, 2), (M // 2, 0, 0), (3, 0, 1)):
        check_select(*x, P, S, first, last)


# ---------------------------------------------------------------------------
# attention

def check_wide(c, M, chunk=None):
    """The requests of case c under a table of M columns, those past their pages naming any."""
    B, m = c.table.shape
    wide = torch.randint(-3, c.mem.shape[0] + 3, (B, M), generator=torch.Generator().manual_seed(M), dtype=torch.int32)
    wide[:, :m] = c.table
    if chunk is not None:                            # how a request's tokens are cut, as the workspace tells
        cache = stepq.Cache(0, c.Hkv, c.P, c.D, c.bits, memory=torch.empty(0, dtype=torch.uint8))
        size = stepq.stepq_cache_attention_workspace(cache, B, c.q.shape[1], M, 0, c.q.dtype)
        assert size == -(-M * c.P // chunk) * B * c.q.shape[1] * (4 * c.D + 8)
    narrow, c.table = c.table, wide
    o, lse = c.call()
    c.table = narrow
    ro, size, rl = C.attention(c.q, c.K, c.V, c.table, c.lengths, None, c.D ** -0.5)
    off = (o.double() - ro).abs()
    bound = 3e-5 * size if o.dtype == F32 else 2.0 ** -14 * size + 2.0 ** -8 * ro.abs()
    assert (off <= bound + 1e-30).all(), ((off - bound) / (size + 1e-30)).max()
    assert torch.equal(torch.isinf(lse), torch.isinf(rl))
    fine = ~torch.isinf(rl)
    assert ((lse.double() - rl).abs()[fine] <= 3e-5 * rl.abs().clamp(min=1.0)[fine]).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("chunk", [384, 640, 1024])
@pytest.mark.parametrize("P", [1, 3, 64])
def test_ranges_of_any_length(P, chunk, bits, act):
    """3 requests x 2 heads under a table of chunk x 512 / 6 tokens: ranges of `chunk` tokens, of up to 1024 pages."""
    c = Case([2 * chunk + 77, chunk, chunk + 1], 4, 2, 64, P, bits, act, seed=P)
    check_wide(c, chunk * 512 // 6 // P if chunk < 1024 else 100000 // P, chunk)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("D", [128, 256])
def test_ranges_of_any_length_of_larger_heads(D, act):
    for bits in (8, 4):
        c = Case([1500, 0, 1025], 6, 2, D, 24, bits, act, seed=D)
        check_wide(c, 100000 // 24, 1024)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_one_range_of_many_pages(bits, act):
    """Pages of one token: more than a workgroup's threads look up at once."""
    n = 700 if act == BF16 else 500
    Case([n, 3, 257], 4, 2, 64, 1, bits, act).check()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("S", [94, 250])
def test_selected_pages_over_several_ranges(S, bits, act):
    """1504 and 4000 tokens of selected pages: 6 and 16 ranges, with keys in each; lists with entries that are no page, and a
    request shorter than most of what it selects."""
    P, M = 16, S + 9
    c = Case([M * P - 5, 300, M * P], 6, 3, 64, P, bits, act, seed=S)
    g = torch.Generator().manual_seed(S)
    sel = torch.stack([torch.randperm(M, generator=g)[:S] for _ in range(9)]).view(3, 3, S).to(torch.int32)
    sel[0, 0, ::7], sel[2, 1, S // 2:], sel[2, 2, 0] = -1, M, 2 ** 31 - 1
    sel[1, 2] = -1
    c.check(selected=sel)


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128])
def test_many_heads_of_a_group_in_several_ranges(D, bits, act):
    Case([3000, 257, 0], 20, 1, D, 16, bits, act).check()
