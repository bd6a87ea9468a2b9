"""64-bit forms of the recurrences and of attention, straight from their
definitions, for the tests of the calls around the decode step."""
import math

import torch

DECAY, DELTA = 0, 1


def recurrence(q, k, v, alpha, beta, S, rule):
    """Tokens [T] of one sequence, all heads: o [T][Hv][dv] and the final state, in float64."""
    q, k, v, alpha = (x.detach().cpu().double() for x in (q, k, v, alpha))
    beta = torch.ones_like(alpha) if beta is None else beta.detach().cpu().double()
    rep = v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    S = S.detach().cpu().double().clone()
    o = torch.empty_like(v)
    for t in range(v.shape[0]):
        S = S * alpha[t][:, None, None]
        u = v[t] - (k[t][:, :, None] * S).sum(1) if rule == DELTA else v[t]
        S = S + k[t][:, :, None] * (beta[t][:, None] * u)[:, None, :]
        o[t] = (q[t][:, :, None] * S).sum(1)
    return o, S


def unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def tokens(T, hv, hqk, dk, dv, act, gate, seed, low=0.95):
    """Decode-like inputs of T tokens on the CPU: q, k, v in act, alpha (low .. 1), beta in gate."""
    g = torch.Generator().manual_seed(seed)
    q, k = (unit(torch.randn((T, hqk, dk), generator=g)).to(act) for _ in range(2))
    v = torch.randn((T, hv, dv), generator=g).to(act)
    alpha = (low + (1 - low) * torch.rand((T, hv), generator=g)).to(gate)
    beta = torch.sigmoid(torch.randn((T, hv), generator=g)).to(gate)
    return q, k, v, alpha, beta


def attention(q, k_cache, v_cache, prefix_pages, prefix_len, table, lengths, scale):
    """o [B][Hq][D], its bound sum_t p_t |v_t|, and lse [B][Hq], in float64."""
    q, kc, vc = (x.detach().cpu().double() for x in (q, k_cache, v_cache))
    B, Hq, D = q.shape
    n_pages, Hkv, page = kc.shape[:3]
    rep = Hq // Hkv
    o, size = torch.zeros(B, Hq, D, dtype=torch.float64), torch.zeros(B, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64)
    for b in range(B):
        at = [(int(prefix_pages[t // page]), t % page) for t in range(prefix_len)]
        n = min(max(int(lengths[b]), 0), table.shape[1] * page)
        at += [(int(table[b, t // page]), t % page) for t in range(n)]
        at = [x for x in at if 0 <= x[0] < n_pages]
        if not at:
            continue
        p, r = (torch.tensor(x) for x in zip(*at))
        K, V = kc[p, :, r], vc[p, :, r]                       # [t][Hkv][D]
        s = torch.einsum("hgd,thd->hgt", q[b].view(Hkv, rep, D), K) * scale
        top = s.amax(-1, keepdim=True)
        w = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        z = w.sum(-1, keepdim=True)
        w = torch.where(z > 0, w / z, torch.zeros_like(w))
        o[b] = torch.einsum("hgt,thd->hgd", w, V).reshape(Hq, D)
        size[b] = torch.einsum("hgt,thd->hgd", w, V.abs()).reshape(Hq, D)
        lse[b] = torch.where(z > 0, top + torch.log(z), torch.full_like(z, -math.inf)).reshape(Hq)
    return o, size, lse
