"""Attention of single tokens over quantized caches, against its definition in
64 bits on the values that the caches hold.

Tolerances.  Codes are exact in the products, queries and (float32) weights have
24 bits, sums are fp32.  float32: scores of up to about 12, each off by a few
2^-24 of what is summed, make the weights off by as much relatively: 3e-5 of
sum_t p_t |v_t|, as for the unquantized call.  bfloat16: the weights have 16 bits
(2^-17 each after two roundings of 8), taken as 2^-14 of sum_t p_t |v_t| with the
scores' share, and the output is rounded once: 2^-8 of it at most.  lse: 3e-5 of
max(1, |lse|)."""
import math

import pytest
import torch

import _cache as C
from paper_2609_38169_amd import stepq

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


class Case:
    """Requests over pages of a cache; what no request's tokens use holds noise (every scale there NaN or infinite)."""

    def __init__(self, lens, Hq, Hkv, D, P, bits, act, seed=1, spare=2, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        M = -(-max(lens, default=0) // P) if max_pages is None else max_pages
        n = B * M + spare
        self.mem, self.K, self.V = C.fill(n, Hkv, P, D, bits, seed)
        self.table = torch.randperm(n, generator=g).to(torch.int32)[:B * M].view(B, M)
        self.lengths = torch.tensor(lens, dtype=torch.int32)
        self.q = (2 * torch.randn((B, Hq, D), generator=g)).to(act)
        self.P, self.D, self.bits, self.Hkv = P, D, bits, Hkv
        used = torch.zeros((n, P), dtype=torch.bool)
        for b in range(B):
            for t in range(min(lens[b], M * P)):
                used[self.table[b, t // P], t % P] = True
        for x in C.parts(self.mem, P, D, bits)[2:]:
            page, row = (~used).nonzero(as_tuple=True)
            x.view(torch.int16)[page, :, row] = 0x7f80 if seed % 2 else 0x7fc0

    def call(self, scale=None, selected=None, stream=None, lse=True, workspace=None):
        cache = stepq.Cache(self.mem.shape[0], self.Hkv, self.P, self.D, self.bits, memory=self.mem.to(DEV).flatten())
        o = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device=DEV)
        L = torch.full(self.q.shape[:2], 7.0, device=DEV) if lse else None
        args = [x.to(DEV) for x in (self.q, self.table, self.lengths)]
        torch.cuda.synchronize()
        cache.attend(*args, o, L, None if selected is None else selected.to(DEV), scale, workspace, stream)
        torch.cuda.synchronize()
        return o.cpu(), None if L is None else L.cpu()

    def check(self, scale=None, selected=None, **kw):
        o, lse = self.call(scale, selected, **kw)
        ro, size, rl = C.attention(self.q, self.K, self.V, self.table, self.lengths, selected,
                                   self.D ** -0.5 if scale is None else scale)
        off = (o.double() - ro).abs()
        bound = 3e-5 * size if o.dtype == F32 else 2.0 ** -14 * size + 2.0 ** -8 * ro.abs()
        assert (off <= bound + 1e-30).all(), ((off - bound) / (size + 1e-30)).max()
        if lse is not None:
            assert torch.equal(torch.isinf(lse), torch.isinf(rl))
            fine = ~torch.isinf(rl)
            assert ((lse.double() - rl).abs()[fine] <= 3e-5 * rl.abs().clamp(min=1.0)[fine]).all()
        return o, lse


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lens", [[1], [0, 1, 31, 32, 33, 65], [300, 2, 0], [128, 129]], ids=lambda x: "-".join(map(str, x)))
def test_lengths(lens, bits, act):
    Case(lens, 8, 2, 128, 16, bits, act).check()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_heads(D, bits, act):
    for Hq, Hkv in ((1, 1), (3, 3), (6, 2), (5, 1), (16, 1), (20, 1), (40, 2)):
        Case([70, 1, 33], Hq, Hkv, D, 16, bits, act, seed=Hq).check()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("G", [2, 4, 5, 8, 9])
def test_scales_of_more_groups(G, D, act):    # 4 bits: 4 or 8 heads and fewer take the matrix cores' columns twice
    Case([70, 1, 33, 0], 2 * G, 2, D, 16, 4, act, seed=G).check()
    Case([1500], G, 1, D, 16, 4, act, seed=G).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("P", [1, 3, 24, 64, 100, 256])
def test_pages(P, bits):
    Case([70, 101, 5], 4, 2, 64, P, bits, BF16, max_pages=-(-101 // P) + 2).check()
    Case([70, 101, 5], 3, 1, 128, P, bits, F32).check()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_in_parts(D, bits, act):
    """Lengths that are split over workgroups, and a request with one token beside them."""
    Case([3000, 1, 1111], 4, 2, D, 64, bits, act).check()


@pytest.mark.parametrize("act", [F32, BF16])
def test_rows_without_a_key(act):
    for mp in (2, 200):                                   # in one part, in several
        c = Case([0, 5, 0, 0], 4, 2, 64, 16, 8, act, max_pages=mp)
        c.lengths[3] = -4
        o, lse = c.check()
        assert not o[0].any() and not o[2:].any() and (lse[0] == -math.inf).all() and (lse[3] == -math.inf).all()
    c = Case([0, 0], 4, 2, 64, 16, 8, act)                # no pages at all
    assert c.table.shape == (2, 0)
    c.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_a_cache_without_a_page(bits):
    c = Case([9, 40], 4, 2, 64, 16, bits, BF16)
    c.mem, c.K, c.V = c.mem[:0], c.K[:0], c.V[:0]
    o, lse = c.check()
    assert not o.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_page_ids_out_of_range_are_left_out(bits):
    c = Case([50, 20, 700], 4, 2, 64, 16, bits, F32)
    c.table[0, 1], c.table[1, 0], c.table[2, 7] = -1, 10 ** 6, c.mem.shape[0]
    c.table[1, 1] = -2 ** 31                              # request 1 has no key left
    c.check()


def test_lengths_past_the_pages_are_cut():
    c = Case([32, 5], 4, 2, 64, 16, 8, BF16)
    c.lengths[0] = 2 ** 31 - 1
    c.check()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("scale", [0.0, 0.5, -0.1])
def test_scales(scale, bits, act):
    c = Case([40, 3, 65], 4, 2, 64, 16, bits, act)
    o, lse = c.call(scale)
    ro, size, rl = C.attention(c.q, c.K, c.V, c.table, c.lengths, None, scale)
    # scores up to about 30 x 2^-22 of D = 64 fp32 terms: the weights' relative error
    tol = 1e-4 if act == F32 else 2.0 ** -13
    assert ((o.double() - ro).abs() <= tol * size + (2.0 ** -8 * ro.abs() if act == BF16 else 0)).all()
    assert ((lse.double() - rl).abs() <= 3e-5 * rl.abs().clamp(min=1.0)).all()


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_keys_and_values_of_any_size(bits, act):
    """Rows whose magnitudes differ by powers of ten, zero rows among them: a key of many times the others' size
    takes all the weight, values of any size are summed as they are."""
    c = Case([50, 20], 4, 2, 64, 16, bits, act)
    g = torch.Generator().manual_seed(5)
    for i, x in ((2, c.K), (3, c.V)):
        f = 2.0 ** torch.randint(-40, 4 if i == 2 else 41, x.shape[:3], generator=g).double()
        f[0::3, :, 1::5] = 0.0
        s = C.parts(c.mem, 16, 64, bits)[i]
        s.view(torch.bfloat16).mul_(f[..., None].to(torch.bfloat16))
        x.mul_(f[..., None])
    o, lse = c.call()
    ro, size, rl = C.attention(c.q, c.K, c.V, c.table, c.lengths, None, 64 ** -0.5)
    # scores up to about 100: the weights' relative error is 100 x 2^-21
    tol = 1e-4 if act == F32 else 2.0 ** -13
    assert ((o.double() - ro).abs() <= tol * size + (2.0 ** -8 * ro.abs() if act == BF16 else 0) + 1e-30).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_not_finite(bits):
    """A key that is not finite makes its heads NaN, a value its group of dimensions, and nothing else."""
    c = Case([40, 40, 40], 4, 2, 128, 16, bits, BF16)
    clean, _ = c.call()
    page, g4 = int(c.table[1, 0]), bits == 4
    C.parts(c.mem, 16, 128, bits)[2].view(torch.int16)[page, 0, 3, 0] = 0x7fc0
    C.parts(c.mem, 16, 128, bits)[3].view(torch.int16)[int(c.table[2, 1]), 1, 2, 0] = 0x7fc0
    o, _ = c.call()
    hit = torch.zeros(o.shape, dtype=torch.bool)
    hit[1, :2] = True
    hit[2, 2:, :64 if g4 else 128] = True
    assert torch.isnan(o[hit]).all() and torch.equal(o[~hit], clean[~hit])


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_selected(bits, act):
    """Each key/value head reads pages of its own, in any order; what is no page of the request's is none."""
    c = Case([100, 37, 600, 0], 6, 3, 64, 16, bits, act)
    g = torch.Generator().manual_seed(4)
    M = c.table.shape[1]
    for S in (1, 3, 20):
        sel = torch.stack([torch.randperm(M, generator=g)[:S] for _ in range(12)]).view(4, 3, S).to(torch.int32)
        sel[0, 0, -1], sel[2, 1, S // 2], sel[2, 2, 0] = -1, M, 2 ** 31 - 1
        sel[1, 2] = -1
        c.check(selected=sel)


@pytest.mark.parametrize("bits", [8, 4])
def test_all_pages_selected(bits):
    """All pages in order are the whole request."""
    c = Case([500, 250], 8, 2, 128, 64, bits, BF16)
    sel = torch.arange(c.table.shape[1], dtype=torch.int32).expand(2, 2, -1).contiguous()
    a, b = c.check(selected=sel), c.check()
    assert ((a[0].double() - b[0].double()).abs() <= 2.0 ** -7 * b[0].double().abs() + 1e-3).all()


def test_many_requests():
    Case([(13 * i) % 41 for i in range(150)], 8, 4, 64, 16, 4, BF16).check()


def test_stream_and_no_lse():
    c = Case([400, 3, 65], 4, 2, 64, 16, 8, BF16)
    a, _ = c.call()
    b, none = c.call(stream=torch.cuda.Stream(), lse=False)
    assert none is None and torch.equal(a, b)


def test_own_workspace():
    c = Case([900, 3, 65], 4, 2, 64, 16, 8, BF16)
    cache = stepq.Cache(c.mem.shape[0], 2, 16, 64, 8)
    n = stepq.stepq_cache_attention_workspace(cache, 3, 4, c.table.shape[1])
    assert n > 0
    a, _ = c.call()
    b, _ = c.call(workspace=torch.full((n,), 255, dtype=torch.uint8, device=DEV))
    assert torch.equal(a, b)


def test_offsets_over_32_bits():
    """Pages beyond 2^32 bytes of the cache."""
    small = Case([100, 20], 16, 8, 256, 256, 8, BF16)
    rec = small.mem.shape[-1]
    n = 2 ** 32 // (8 * rec) + 20
    cache = stepq.Cache(n, 8, 256, 256, 8)
    ids = torch.tensor([n - 1, n - 9, 0, 7][:small.mem.shape[0]])
    cache.memory.view(n, 8, rec)[ids.to(DEV)] = small.mem.to(DEV)
    o = torch.empty_like(small.q, device=DEV)
    cache.attend(small.q.to(DEV), ids[small.table.long()].to(torch.int32).to(DEV), small.lengths.to(DEV), o)
    ro, size, _ = C.attention(small.q, small.K, small.V, small.table, small.lengths, None, 1 / 16)
    assert ((o.cpu().double() - ro).abs() <= 2.0 ** -14 * size + 2.0 ** -8 * ro.abs()).all()


def test_refusals():
    c = Case([50, 20], 4, 2, 64, 16, 8, BF16)
    cache = stepq.Cache(c.mem.shape[0], 2, 16, 64, 8, memory=c.mem.to(DEV).flatten())
    q, table, lengths = (x.to(DEV) for x in (c.q, c.table, c.lengths))
    o = torch.empty_like(q)
    sel = torch.zeros((2, 2, 3), dtype=torch.int32, device=DEV)
    f = cache.attend
    with pytest.raises(TypeError):
        f(q.half(), table, lengths, o)
    with pytest.raises(TypeError):
        f(q, table, lengths, o.float())
    with pytest.raises(ValueError):
        f(q[:, :, :32].contiguous(), table, lengths, o)
    with pytest.raises(ValueError):
        f(q.transpose(0, 1), table, lengths, o)
    with pytest.raises(ValueError):
        f(q[:1], table, lengths, o)
    with pytest.raises(TypeError):
        f(q, table.long(), lengths, o)
    with pytest.raises(ValueError):
        f(q, table, lengths[:1], o)
    with pytest.raises(ValueError):
        f(q, table, lengths, o, selected=sel[:, :1])
    with pytest.raises(ValueError):
        f(q, table, lengths, o, selected=sel[:, :, :0])
    with pytest.raises(TypeError):
        f(q, table, lengths, o, selected=sel.long())
    with pytest.raises(stepq.StepqError):
        f(q, table, lengths, o, scale=math.inf)
    with pytest.raises(stepq.StepqError):
        f(q[:, :3].contiguous(), table, lengths, o[:, :3].contiguous())
    with pytest.raises((ValueError, TypeError)):
        f(q, table, lengths, o, workspace=torch.empty(4, device=DEV))
    with pytest.raises(ValueError):
        f(q.cpu(), table, lengths, o)
