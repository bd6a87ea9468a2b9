"""What a serving program asks around the decode step of the state pool, as timed cases.

A request reaches the pool through its prompt; its state may be advanced
before it is quantized; and the models whose recurrent layers the pool serves
have full-attention layers between them, whose cache a batch with a common
prefix reads once.  The cases, at head sizes and counts of the workloads in
paper_2609_38169_amd/workloads.py and of the tests, or generic ones:

  kind "prompt"  linear attention over packed prompts, from given or empty
                 states to the outputs of every token and the final states;
                 rule "decay" or "delta"; `n_seq` prompts of len_min ..
                 len_max tokens; shared: every prompt starts from one common
                 state (a prefix done before), else from zeros; fused: q, k and
                 v are slices of one projection's output
  kind "step"    the same recurrences for one token of `batch` requests, on
                 full-precision states updated in place
  kind "attn"    softmax attention of one token of `batch` requests over a
                 common prefix of `prefix` tokens and 1 .. own tokens of each
                 request's own, keys and values in pages of `page` tokens

act "f32" or "bf16" is the type of the activations, caches and outputs.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
CHUNK = 64


def _prompt(name, **kw):
    c = dict(name=name, kind="prompt", rule="delta", n_seq=1, len_min=1, len_max=1, hv=32, hqk=16, dk=128, dv=128,
             act="bf16", shared=False, fused=False)
    c.update(kw)
    return c


def _step(name, **kw):
    c = dict(name=name, kind="step", rule="delta", n_states=0, batch=1, hv=32, hqk=16, dk=128, dv=128, act="bf16")
    c.update(kw)
    c["n_states"] = c["n_states"] or c["batch"]
    return c


def _attn(name, **kw):
    c = dict(name=name, kind="attn", batch=1, hq=16, hkv=2, d=128, prefix=0, own=1, page=16, act="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # one user's few parallel samples of a short system prompt: latency
        _attn("attn_b4", batch=4, hq=8, hkv=2, prefix=512, own=64),
        # medium concurrency, long answers: the requests' own caches are most of the bytes
        _attn("attn_b64", batch=64, hq=32, hkv=8, prefix=4096, own=1024),
        # high concurrency over a long document: the prefix is a matrix product
        _attn("attn_b512", batch=512, hq=16, hkv=2, d=256, prefix=16384, own=256, page=64),
        # odd sizes: a prefix and pages that end inside any tile, 3 query heads a group, fp32
        _attn("attn_odd_f32", batch=23, hq=12, hkv=4, d=64, prefix=1001, own=333, page=24, act="f32"),
        # one token of one request on a small model: latency
        _step("step_tiny", rule="decay", hv=4, hqk=4, dk=64, dv=64, act="f32"),
        # a whole layer's states kept in full precision: memory only
        _step("step_b512", batch=512, n_states=640),
        # one long document through a layer with per-head decay
        _prompt("decay_long", rule="decay", len_min=32768, len_max=32768, hqk=32),
        # short prompts on a small fp32 model, no size a power of two
        _prompt("decay_odd_f32", rule="decay", n_seq=24, len_min=1, len_max=700, hv=6, hqk=3, dk=96, dv=64, act="f32"),
        # one request's prompt on a gated-Delta layer, time to first token
        _prompt("delta_one", len_min=8192, len_max=8192, fused=True),
        # the prompts of a batch before their states are packed into the pool
        _prompt("delta_b32", n_seq=32, len_min=128, len_max=2048, fused=True),
        # a batch's own short prompts after a common prefix
        _prompt("delta_shared", n_seq=64, len_min=1, len_max=200, shared=True),
        # the same rule on a small fp32 model with odd head sizes
        _prompt("delta_odd_f32", n_seq=5, len_min=1, len_max=1500, hv=6, hqk=3, dk=77, dv=64, act="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt"] * 5 + ["attn"] * 4 + ["step"])
    act = rng.choice(["bf16", "bf16", "f32"])
    if kind == "attn":
        hkv = rng.choice([1, 2, 4, 8])
        d = rng.choice([64, 128, 128, 256])
        hq = min(hkv * rng.choice([1, 2, 3, 4, 5, 8, 16]), 32)
        hq -= hq % hkv
        b = _log(rng, 1, 400 if act == "bf16" else 64)
        # queries x keys at most those of the largest listed case
        prefix = min(_log(rng, 1, 32768), (512 * 16 * 16384 * 256) // (b * hq * d))
        if act == "f32":
            prefix = min(prefix, 8192)
        mine = min(_log(rng, 1, 4096), max(1, 2 ** 27 // (b * hkv * d)))
        return _no_name(_attn("", batch=b, hq=hq, hkv=hkv, d=d, prefix=prefix if rng.random() < 0.9 else 0, own=mine,
                              page=rng.choice([1, 16, 16, 24, 32, 64, 100, 256]), act=act))
    rule = rng.choice(["delta", "delta", "decay"])
    hqk = rng.choice([1, 2, 4, 8, 16])
    hv = min(32, hqk * rng.choice([1, 1, 2, 3]))
    hv -= hv % hqk
    dk, dv = rng.choice([(128, 128)] * 4 + [(64, 64), (96, 128), (77, 64), (128, 64), (37, 128)])
    if kind == "step":
        b = _log(rng, 1, 512)
        return _no_name(_step("", rule=rule, batch=b, n_states=b + rng.randrange(0, 9), hv=hv, hqk=hqk, dk=dk, dv=dv,
                              act=act))
    total = _log(rng, 64, 40000)                       # tokens of all prompts together, at most
    n = min(_log(rng, 1, 96), total)
    top = min(max(1, total // n), 32768 if rule == "decay" else 8192)
    return _no_name(_prompt("", rule=rule, n_seq=n, len_min=rng.choice([1, top, max(1, top // 4)]), len_max=top, hv=hv,
                            hqk=hqk, dk=dk, dv=dv, act=act, shared=rng.random() < 0.3, fused=rng.random() < 0.4))


def _no_name(c):
    c.pop("name")
    return c


# ---------------------------------------------------------------------------
# inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + stream) & ((1 << 62) - 1))
    return g


def _dtype(c):
    return torch.bfloat16 if c["act"] == "bf16" else torch.float32


def lengths(c):
    """Tokens of each prompt, or of each request's own cache: the traffic a case stands for, the same for every seed."""
    if c["kind"] == "attn":
        return np.random.default_rng([c["batch"], c["own"]]).integers(1, c["own"] + 1, c["batch"])
    return np.random.default_rng([c["n_seq"], c["len_max"]]).integers(c["len_min"], c["len_max"] + 1, c["n_seq"])


def _unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def _activations(c, seed, T):
    """q, k (unit norm), v, alpha, beta of T tokens, as the decode step's inputs are distributed."""
    g, dt = _gen(seed, 1), _dtype(c)
    q = _unit(torch.randn((T, c["hqk"], c["dk"]), generator=g, device=DEV)).to(dt)
    k = _unit(torch.randn((T, c["hqk"], c["dk"]), generator=g, device=DEV)).to(dt)
    v = torch.randn((T, c["hv"], c["dv"]), generator=g, device=DEV).to(dt)
    alpha = 1.0 - 0.05 * torch.rand((T, c["hv"]), generator=g, device=DEV)
    beta = torch.sigmoid(torch.randn((T, c["hv"]), generator=g, device=DEV))
    if c.get("fused"):
        nq, nv = c["hqk"] * c["dk"], c["hv"] * c["dv"]
        x = torch.cat([q.reshape(T, nq), k.reshape(T, nq), v.reshape(T, nv)], 1)
        q, k = x[:, :nq].view(T, c["hqk"], c["dk"]), x[:, nq:2 * nq].view(T, c["hqk"], c["dk"])
        v = x[:, 2 * nq:].view(T, c["hv"], c["dv"])
    return q, k, v, alpha, beta


def _states(c, seed, n):
    return 0.05 * torch.randn((n, c["hv"], c["dk"], c["dv"]), generator=_gen(seed, 2), device=DEV)


def prepare(c, seed):
    if c["kind"] == "attn":
        return _prepare_attn(c, seed)
    s = dict(case=c)
    if c["kind"] == "step":
        B = c["batch"]
        s["act"] = _activations(c, seed, B)
        s["state"] = _states(c, seed, c["n_states"])
        s["ids"] = torch.randperm(c["n_states"], generator=_gen(seed, 3), device=DEV)[:B].to(torch.int32)
        s["o"] = torch.zeros((B, c["hv"], c["dv"]), device=DEV)
        return s
    ends = np.concatenate([[0], np.cumsum(lengths(c))])
    T, n = int(ends[-1]), c["n_seq"]
    s["cu"] = torch.from_numpy(ends.astype(np.int32)).to(DEV)
    s["act"] = _activations(c, seed, T)
    s["start"] = _states(c, seed, 1) if c["shared"] else None
    s["ids"] = torch.zeros(n, dtype=torch.int32, device=DEV) if c["shared"] else None
    s["o"] = torch.zeros((T, c["hv"], c["dv"]), dtype=_dtype(c), device=DEV)
    s["state"] = torch.zeros((n, c["hv"], c["dk"], c["dv"]), device=DEV)
    return s


def _prepare_attn(c, seed):
    g, dt, B, page = _gen(seed, 4), _dtype(c), c["batch"], c["page"]
    n_pre, n_own = -(-c["prefix"] // page), -(-c["own"] // page)
    n_pages = n_pre + B * n_own + 3
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(dt)
    # some keys point where some queries do, as in a trained model: scores up to about 8 after the scale
    s = dict(case=c, q=rnd(B, c["hq"], c["d"]) * 2, k=rnd(n_pages, c["hkv"], page, c["d"]),
             v=rnd(n_pages, c["hkv"], page, c["d"]))
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    s["prefix_pages"] = ids[:n_pre].contiguous()
    s["table"] = ids[n_pre:n_pre + B * n_own].view(B, n_own).contiguous()
    s["lengths"] = torch.from_numpy(lengths(c).astype(np.int32)).to(DEV)
    s["o"] = torch.zeros((B, c["hq"], c["d"]), dtype=dt, device=DEV)
    s["lse"] = torch.zeros((B, c["hq"]), device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    if own:
        from paper_2609_38169_amd import stepq
        rule = stepq.STEPQ_RULE_DELTA if c.get("rule") == "delta" else stepq.STEPQ_RULE_DECAY
        if c["kind"] == "attn":
            stepq.stepq_prefix_attention(s["q"], s["k"], s["v"], s["prefix_pages"], c["prefix"], s["table"], s["lengths"],
                                         s["o"], s["lse"])
            return {"o": s["o"], "lse": s["lse"]}
        if c["kind"] == "step":
            stepq.stepq_state_step(s["state"], s["ids"], *s["act"], s["o"], rule)
        else:
            stepq.stepq_prompt(*s["act"], s["o"], s["state"], rule, cu_seqlens=s["cu"], state_in=s["start"],
                               in_ids=s["ids"])
        return {"o": s["o"], "state": s["state"]}
    return {"attn": _attn_plain, "step": _step_plain, "prompt": _prompt_plain}[c["kind"]](s)


def _step_plain(s):
    c = s["case"]
    q, k, v, alpha, beta = (x.float() for x in s["act"])
    rep = c["hv"] // c["hqk"]
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    ids = s["ids"].long()
    S = s["state"][ids] * alpha[..., None, None]
    u = v
    if c["rule"] == "delta":
        u = v - torch.matmul(k[:, :, None, :], S)[:, :, 0]
    S = S + k[..., None] * (beta[..., None] * u)[:, :, None, :]
    s["state"][ids] = S
    return {"o": torch.matmul(q[:, :, None, :], S)[:, :, 0], "state": s["state"]}


def _prompt_plain(s):
    c, cu = s["case"], s["cu"].long()
    n, hv, C = c["n_seq"], c["hv"], CHUNK
    nc = -(-c["len_max"] // C)
    rep = hv // c["hqk"]
    # prompts padded to whole chunks, [n][hv][nc][C][...]; padding has k = v = q = 0 and alpha = 1
    pos = cu[:-1, None] + torch.arange(nc * C, device=cu.device)
    valid = pos < cu[1:, None]
    pos = torch.where(valid, pos, torch.zeros_like(pos))

    def pad(x, fill):
        x = x.float()[pos]
        x = torch.where(valid.view(valid.shape + (1,) * (x.dim() - 2)), x, torch.full_like(x, fill))
        x = x.view((n, nc, C) + x.shape[2:])
        return x.permute((0, 3, 1, 2) + ((4,) if x.dim() == 5 else ())).contiguous()

    q, k, v, alpha, beta = (pad(x, f) for x, f in zip(s["act"], (0.0, 0.0, 0.0, 1.0, 0.0)))
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    G = torch.cumsum(torch.log(alpha), -1)                          # log of the decay since the chunk's start
    D = torch.exp(torch.tril(G[..., :, None] - G[..., None, :]))    # decay from token j to token i
    keep = torch.tril(torch.ones((C, C), dtype=torch.bool, device=cu.device))
    D = torch.where(keep, D, torch.zeros_like(D))
    last = torch.exp(G[..., -1:])
    w = torch.exp(G[..., -1:] - G)                                  # decay from token j to the chunk's end
    G = torch.exp(G)
    P = torch.matmul(q, k.transpose(-1, -2).contiguous()) * D
    if c["rule"] == "delta":
        M = torch.tril(torch.matmul(k, k.transpose(-1, -2).contiguous()) * D * beta[..., None], -1)
        T = torch.eye(C, device=cu.device).expand(M.shape).clone()
        for i in range(1, C):                                       # (I + M) T = I, row by row
            T[..., i, :i] -= torch.matmul(M[..., i, None, :i], T[..., :i, :i])[..., 0, :]
    v = v * beta[..., None]
    if s["start"] is None:
        S = torch.zeros((n, hv, c["dk"], c["dv"]), device=cu.device)
    else:
        S = s["start"][s["ids"].long()]
    o = torch.empty_like(v)
    for i in range(nc):
        U = v[:, :, i]
        if c["rule"] == "delta":
            U = U - torch.matmul(k[:, :, i] * (beta * G)[:, :, i, :, None], S)
            U = torch.matmul(T[:, :, i], U)
        o[:, :, i] = torch.matmul(q[:, :, i] * G[:, :, i, :, None], S) + torch.matmul(P[:, :, i], U)
        kw = (k[:, :, i] * w[:, :, i, :, None]).transpose(-1, -2).contiguous()
        S = S * last[:, :, i, :, None] + torch.matmul(kw, U)
    o = o.permute(0, 2, 3, 1, 4).reshape(n, nc * C, hv, c["dv"])
    return {"o": o[valid].to(s["o"].dtype), "state": S}


def _attn_plain(s):
    c = s["case"]
    B, hq, hkv, d, page = c["batch"], c["hq"], c["hkv"], c["d"], c["page"]
    g, n_own = hq // hkv, s["table"].shape[1]
    q = s["q"].float().view(B, hkv, g, d) * d ** -0.5
    qp = q.permute(1, 0, 2, 3).reshape(hkv, B * g, d)
    # the common prefix: [hkv][tokens][d], scores [hkv][B * g][tokens]
    pages = s["prefix_pages"].long()
    kp = s["k"][pages].float().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :c["prefix"]]
    vp = s["v"][pages].float().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :c["prefix"]]
    sp = torch.matmul(qp, kp.transpose(1, 2).contiguous()).view(hkv, B, g, -1).permute(1, 0, 2, 3)
    # each request's own tokens: [B][hkv][tokens][d], scores [B][hkv][g][tokens]
    table = s["table"].long()
    ko = s["k"][table].float().permute(0, 2, 1, 3, 4).reshape(B, hkv, n_own * page, d)
    vo = s["v"][table].float().permute(0, 2, 1, 3, 4).reshape(B, hkv, n_own * page, d)
    so = torch.matmul(q, ko.transpose(2, 3).contiguous())
    valid = torch.arange(n_own * page, device=q.device) < s["lengths"][:, None]
    so = torch.where(valid[:, None, None, :], so, torch.full_like(so, -math.inf))
    m = so.amax(-1)
    if c["prefix"]:
        m = torch.maximum(m, sp.amax(-1))
    ep, eo = torch.exp(sp - m[..., None]), torch.exp(so - m[..., None])
    z = ep.sum(-1) + eo.sum(-1)
    vo = torch.where(valid[:, None, :, None], vo, torch.zeros_like(vo))
    a = torch.matmul(ep.permute(1, 0, 2, 3).reshape(hkv, B * g, -1), vp).view(hkv, B, g, d).permute(1, 0, 2, 3)
    a = (a + torch.matmul(eo, vo)) / z[..., None]
    return {"o": a.reshape(B, hq, d).to(s["o"].dtype), "lse": (m + torch.log(z)).reshape(B, hq)}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(c):
    a = 2 if c["act"] == "bf16" else 4
    n = lengths(c) if c["kind"] != "step" else None
    if c["kind"] == "attn":
        mine = int(n.sum())
        return {"bytes": 2.0 * a * c["hkv"] * c["d"] * (c["prefix"] + mine)
                + c["batch"] * c["hq"] * (2.0 * a * c["d"] + 4),
                "flops": 4.0 * c["hq"] * c["d"] * (c["batch"] * c["prefix"] + mine)}
    T = c["batch"] if c["kind"] == "step" else int(n.sum())
    el = c["hv"] * c["dk"] * c["dv"]
    per = a * (2 * c["hqk"] * c["dk"] + c["hv"] * c["dv"]) + 8 * c["hv"]
    flops = T * el * (7.0 if c["rule"] == "delta" else 5.0)
    if c["kind"] == "step":
        return {"bytes": T * (8.0 * el + per + 4 * c["hv"] * c["dv"]), "flops": flops}
    start = 4.0 * el if c["shared"] else 0.0
    return {"bytes": T * (per + float(a) * c["hv"] * c["dv"]) + 4.0 * el * c["n_seq"] + start, "flops": flops}


# ---------------------------------------------------------------------------
# the same in 64 bits: token by token, key by key

def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "attn":
        return _attn_exact(c, s)
    q, k, v, alpha, beta = (x.double() for x in s["act"])
    head = torch.arange(c["hv"], device=DEV) // (c["hv"] // c["hqk"])
    delta = c["rule"] == "delta"

    def advance(S, t):
        """States S of some (request, head)s after the tokens t, and what they read: the recurrence itself."""
        kt, qt = k[t][:, head], q[t][:, head]
        S = S * alpha[t][..., None, None]
        u = v[t] - (torch.matmul(kt.unsqueeze(2), S).squeeze(2) if delta else 0.0)
        S = S + kt.unsqueeze(3) * (beta[t].unsqueeze(2) * u).unsqueeze(2)
        return S, torch.matmul(qt.unsqueeze(2), S).squeeze(2)

    if c["kind"] == "step":
        ids = s["ids"].long()
        state = s["state"].double()
        state[ids], o = advance(state[ids], torch.arange(c["batch"], device=DEV))
        return {"o": o, "state": state}
    n = lengths(c)
    if int(n.max()) * max(1.0, c["n_seq"] * c["hv"] * c["dk"] * c["dv"] / 2e6) > 6e4:
        return None
    first = np.concatenate([[0], np.cumsum(n)])[:-1]
    o = torch.empty((int(n.sum()), c["hv"], c["dv"]), dtype=torch.float64, device=DEV)
    state = torch.zeros((c["n_seq"], c["hv"], c["dk"], c["dv"]), dtype=torch.float64, device=DEV)
    if c["shared"]:
        state += s["start"].double()
    order = np.argsort(-n, kind="stable")                # longest first: those still running are a leading part
    at = torch.from_numpy(first[order]).to(DEV)
    back = torch.from_numpy(order).to(DEV)
    state = state[back]
    for t in range(int(n.max())):
        live = int((n > t).sum())
        state[:live], o[at[:live] + t] = advance(state[:live], at[:live] + t)
    out = torch.empty_like(state)
    out[back] = state
    return {"o": o, "state": out}


def _attn_exact(c, s):
    B, hq, d, page = c["batch"], c["hq"], c["d"], c["page"]
    g = hq // c["hkv"]
    pre = torch.arange(c["prefix"], device=DEV)
    pre_page, pre_row = s["prefix_pages"].long()[pre // page], pre % page
    n = lengths(c)
    o = torch.empty((B, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, hq), dtype=torch.float64, device=DEV)
    kp, vp = (x[pre_page, :, pre_row].double().transpose(0, 1) for x in (s["k"], s["v"]))     # [hkv][prefix][d]
    for b in range(B):
        t = torch.arange(int(n[b]), device=DEV)
        at = s["table"][b].long()[t // page]
        kb = torch.cat([kp, s["k"][at, :, t % page].double().transpose(0, 1)], 1)
        vb = torch.cat([vp, s["v"][at, :, t % page].double().transpose(0, 1)], 1)
        x = (s["q"][b].double().view(c["hkv"], g, 1, d) * kb[:, None]).sum(-1) / math.sqrt(d) if d * g * kb.shape[1] < 2 ** 16 \
            else torch.bmm(s["q"][b].double().view(c["hkv"], g, d), kb.transpose(1, 2).contiguous()) / math.sqrt(d)
        lse[b] = torch.logsumexp(x, -1).view(hq)
        o[b] = torch.bmm(torch.softmax(x, -1), vb).view(hq, d)
    return {"o": o, "lse": lse}
