"""Quantized key/value caches from their definition (include/stepq.h), in 64
bits on the CPU, for the tests of the calls on them."""
import math

import torch

TOP = {8: 127.0, 4: 7.0}


def scales_per_row(D, bits):
    return 1 if bits == 8 else D // 64


def record_bytes(P, D, bits):
    return -(-2 * P * (D * bits // 8 + 2 * scales_per_row(D, bits)) // 128) * 128


def bf16_up(x):
    """The smallest bfloat16 that is not below x >= 0 (float64), as float64."""
    f, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), torch.clamp(e - 8, min=-133).to(torch.float64))
    return torch.ceil(x / step) * step


def quantize(x, bits):
    """Whole codes and scales (both float64) of rows x [..., D]."""
    x = x.detach().cpu().double()
    D, top = x.shape[-1], TOP[bits]
    x = x.unflatten(-1, (scales_per_row(D, bits), -1))
    a = x.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(a)
    y = torch.where(fine, a, torch.zeros_like(a))
    s = bf16_up(y / top)
    # y / top is rounded: the definition itself, a step either way
    f, e = torch.frexp(torch.where(s > 0, s, torch.ones_like(s)))
    step = torch.ldexp(torch.ones_like(s), torch.clamp(e - 8, min=-133).to(torch.float64))
    s = torch.where((s - step) * top >= y, s - step, s)
    s = torch.where(s * top < y, s + step, s)
    s = torch.where(y < 2.0 ** -100, torch.zeros_like(s), s)
    c = torch.where(s > 0, torch.round(x / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(x))
    c = torch.where(fine, c, torch.zeros_like(c))
    s = torch.where(fine, s, torch.full_like(s, math.nan))
    return c.flatten(-2), s[..., 0]


def value(c, s):
    return c * s.repeat_interleave(c.shape[-1] // s.shape[-1], -1)


def held(x, bits):
    """What a cache holds of rows x."""
    return value(*quantize(x, bits))


def rows_to_bytes(c, bits):
    c = c.to(torch.int32)
    if bits == 8:
        return (c & 255).to(torch.uint8)
    D = c.shape[-1]
    out = torch.zeros(c.shape[:-1] + (D // 2,), dtype=torch.int32)
    for w in range(D // 4):
        for j in range(4):
            out[..., 2 * w + j // 2] |= (c[..., D // 4 * j + w] & 15) << 4 * (j % 2)
    return out.to(torch.uint8)


def scales_to_bytes(s):
    return s.to(torch.bfloat16).contiguous().view(torch.uint8)


def parts(mem, P, D, bits):
    """Views [n_pages][Hkv][P][...] of a cache's bytes [n_pages][Hkv][record]: key codes, value codes, key scales, value scales."""
    rb, sb = D * bits // 8, 2 * scales_per_row(D, bits)
    out, at = [], 0
    for n in (rb, rb, sb, sb):
        out.append(mem[..., at:at + P * n].unflatten(-1, (P, n)))
        at += P * n
    return out


def put(mem, P, D, bits, page, row, k, v):
    """Rows k, v [Hkv][D] of one token into a cache's bytes."""
    for i, x in ((0, k), (1, v)):
        c, s = quantize(x, bits)
        parts(mem, P, D, bits)[i][page, :, row] = rows_to_bytes(c, bits)
        parts(mem, P, D, bits)[2 + i][page, :, row] = scales_to_bytes(s)


def fill(n_pages, Hkv, P, D, bits, seed, gain=None):
    """A cache's bytes with a token in every row, and the held keys and values [n_pages][Hkv][P][D]."""
    g = torch.Generator().manual_seed(seed)
    mem = torch.randint(0, 256, (n_pages, Hkv, record_bytes(P, D, bits)), generator=g, dtype=torch.uint8)
    kv = []
    for i in range(2):
        x = torch.randn((n_pages, Hkv, P, D), generator=g)
        if gain is not None and i == 0:
            x = x * gain
        c, s = quantize(x, bits)
        parts(mem, P, D, bits)[i][:] = rows_to_bytes(c, bits)
        parts(mem, P, D, bits)[2 + i][:] = scales_to_bytes(s)
        kv.append(value(c, s))
    return mem, kv[0], kv[1]


def places(table, starts, cu, P, n_pages):
    """(token, page, row) of every token that has a place, and the tokens that lie in a sequence."""
    out, inside = [], []
    n = table.shape[0]
    for i in range(n):
        first, end = (i, i + 1) if cu is None else (int(cu[i]), int(cu[i + 1]))
        for t in range(first, end):
            inside.append(t)
            pos = int(starts[i]) + t - first
            if int(starts[i]) < 0 or pos >= table.shape[1] * P:
                continue
            page = int(table[i, pos // P])
            if 0 <= page < n_pages:
                out.append((t, page, pos % P))
    return out, inside


def attention(q, K, V, table, lengths, selected, scale):
    """o, its bound sum_t p_t |v_t| and lse of one token of each request over held keys and values, in float64."""
    q = q.detach().cpu().double()
    B, Hq, D = q.shape
    n_pages, Hkv, P = K.shape[:3]
    G = Hq // Hkv
    o, size = torch.zeros(B, Hq, D, dtype=torch.float64), torch.zeros(B, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * P)
        for h in range(Hkv):
            pos = range(table.shape[1]) if selected is None else [int(x) for x in selected[b, h]]
            at = [(int(table[b, p]), max(0, min(P, n - p * P))) for p in pos if 0 <= p < table.shape[1]]
            at = [x for x in at if 0 <= x[0] < n_pages and x[1]]
            if not at:
                continue
            k, v = (torch.cat([x[page, h, :m] for page, m in at]) for x in (K, V))
            s = q[b, h * G:(h + 1) * G] @ k.T * scale
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            z = w.sum(-1, keepdim=True)
            w = torch.where(z > 0, w / z, torch.zeros_like(w)) if not torch.isnan(z).any() else w / z
            o[b, h * G:(h + 1) * G], size[b, h * G:(h + 1) * G] = w @ v, w @ v.abs()
            lse[b, h * G:(h + 1) * G] = torch.where(z == 0, torch.full_like(z, -math.inf), top + torch.log(z))[:, 0]
    return o, size, lse


def bounds_of(k):
    """Bounds [2][D] (bfloat16) of keys k [t][D]."""
    lo, hi = k.amin(0), k.amax(0)                    # a NaN stays one

    def down(x):                                     # to 8 significant bits, towards -inf
        f, e = torch.frexp(torch.where(torch.isnan(x), torch.zeros_like(x), x))
        y = torch.ldexp(torch.floor(f * 256) / 256, e.to(torch.float64))
        return torch.where(torch.isnan(x), x, y)
    return torch.stack([down(lo), -down(-hi)]).to(torch.bfloat16)


def select(q, bounds, table, lengths, P, S, first, last):
    """selected [B][Hkv][S] by the definition of the scores."""
    q, bounds = q.detach().cpu().double(), bounds.cpu().double()
    B, Hq, D = q.shape
    n_pages, Hkv = bounds.shape[:2]
    G = Hq // Hkv
    out = torch.full((B, Hkv, S), -1, dtype=torch.int32)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * P)
        pages = -(-n // P)
        for h in range(Hkv):
            if pages <= S:
                out[b, h, :pages] = torch.arange(pages, dtype=torch.int32)
                continue
            x = q[b, h * G:(h + 1) * G]
            up, down = x.clamp(min=0).sum(0), x.clamp(max=0).sum(0)
            mid = list(range(first, pages - last))
            ids = table[b, first:pages - last].long()
            ok = (ids >= 0) & (ids < n_pages)
            w = bounds[ids.clamp(0, n_pages - 1), h]
            score = (w[:, 1] * up + w[:, 0] * down).sum(-1).float()
            rank = [(0 if not o else 1, math.inf if math.isnan(s) else s, math.isnan(s)) for o, s in zip(ok.tolist(), score.tolist())]
            order = sorted(range(len(mid)), key=lambda i: (-rank[i][0], not rank[i][2], -rank[i][1], i))
            best = sorted(mid[i] for i in order[:S - first - last])
            out[b, h] = torch.tensor(list(range(first)) + best + list(range(pages - last, pages)), dtype=torch.int32)
    return out
