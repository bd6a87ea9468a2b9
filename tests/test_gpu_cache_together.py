"""The calls on quantized caches as a serving program makes them: prompts in
chunks, then decoding with pages selected, step by step against the definitions;
the same captured into graphs; and the example that serves with them.

Tolerances: those of test_gpu_cache_attention.py for attention, none for what is
held, bounds and selections."""
import importlib.util
import os

import pytest
import torch

import _cache as C
from paper_2609_38169_amd import stepq

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("bits", [8, 4])
def test_prompts_then_decoding(bits, act):
    Hq, Hkv, D, P, M, S = 6, 2, 128, 8, 12, 5
    chunks, steps = [[30, 0, 13], [11, 5, 1]], 4
    B, n_pages = 3, 3 * M + 2
    g = torch.Generator().manual_seed(bits)
    rnd = lambda *s: torch.randn(s, generator=g).to(act)
    cache = stepq.Cache(n_pages, Hkv, P, D, bits)
    table = torch.randperm(n_pages, generator=g).to(torch.int32)[:B * M].view(B, M)
    bounds = torch.zeros((n_pages, Hkv, 2, D), dtype=BF16, device=DEV)
    K, V = (torch.zeros((n_pages, Hkv, P, D), dtype=torch.float64) for _ in range(2))
    lens, dt = [0] * B, table.to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)

    def note(b, k, v):                        # a token of request b, as the cache holds it
        page, row = int(table[b, lens[b] // P]), lens[b] % P
        K[page, :, row], V[page, :, row] = C.held(k, bits), C.held(v, bits)
        lens[b] += 1

    def check(q, sel=None):
        o, lse = torch.zeros_like(q, device=DEV), torch.zeros(q.shape[:2], device=DEV)
        cache.attend(q.to(DEV), dt, i32(lens).to(DEV), o, lse, None if sel is None else sel.to(DEV))
        ro, size, rl = C.attention(q, K, V, table, i32(lens), sel, D ** -0.5)
        bound = 3e-5 * size if act == F32 else 2.0 ** -14 * size + 2.0 ** -8 * ro.abs()
        assert ((o.cpu().double() - ro).abs() <= bound + 1e-30).all()
        fine = ~torch.isinf(rl)
        assert ((lse.cpu().double() - rl).abs()[fine] <= 3e-5 * rl.abs().clamp(min=1.0)[fine]).all()

    for n in chunks:
        starts, cu = i32(lens), i32([0] + n).cumsum(0, dtype=torch.int32)
        k, v = rnd(sum(n), Hkv, D), rnd(sum(n), Hkv, D)
        cache.write(k.to(DEV), v.to(DEV), dt, starts.to(DEV), cu.to(DEV))
        for b in range(B):
            for t in range(int(cu[b]), int(cu[b + 1])):
                note(b, k[t], v[t])
        cache.bounds(dt, starts.to(DEV), i32(lens).to(DEV), bounds)
        check(rnd(B, Hq, D))
    back = [torch.zeros((sum(lens), Hkv, D), dtype=act, device=DEV) for _ in range(2)]
    cu = i32([0] + lens).cumsum(0, dtype=torch.int32)
    cache.read(dt, torch.zeros_like(i32(lens)).to(DEV), *back, cu.to(DEV))
    for b in range(B):
        for x, held in zip(back, (K, V)):
            want = held[table[b].long()].transpose(1, 2).reshape(M * P, Hkv, D)[:lens[b]].to(act)
            assert torch.equal(x[int(cu[b]):int(cu[b + 1])].cpu(), want)
    for _ in range(steps):
        starts = i32(lens)
        k, v, q = rnd(B, Hkv, D), rnd(B, Hkv, D), rnd(B, Hq, D)
        cache.write(k.to(DEV), v.to(DEV), dt, starts.to(DEV))
        for b in range(B):
            note(b, k[b], v[b])
        cache.bounds(dt, starts.to(DEV), i32(lens).to(DEV), bounds)
        for b in range(B):
            for p in range(-(-lens[b] // P)):
                page, n = int(table[b, p]), min(P, lens[b] - p * P)
                for h in range(Hkv):
                    assert torch.equal(bounds[page, h].cpu(), C.bounds_of(K[page, h, :n]))
        sel = torch.zeros((B, Hkv, S), dtype=torch.int32, device=DEV)
        cache.select(q.to(DEV), bounds, dt, i32(lens).to(DEV), sel)
        assert torch.equal(sel.cpu(), C.select(q, bounds, table, i32(lens), P, S, 1, 1))
        check(q, sel.cpu())


def decode_state(B=5, Hq=8, Hkv=2, D=64, P=4, M=300, bits=8, seed=1):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g).to(BF16).to(DEV)
    n = B * M
    cache = stepq.Cache(n, Hkv, P, D, bits)
    cache.memory.zero_()                     # rows without a token too: two caches are compared as a whole
    table = torch.randperm(n, generator=g).to(torch.int32).view(B, M).to(DEV)
    lengths = torch.tensor([1, 700, 33, 1100, 64][:B], dtype=torch.int32, device=DEV)
    T = int(lengths.sum())
    cu = torch.cat([lengths.new_zeros(1), lengths.cumsum(0, dtype=torch.int32)])
    cache.write(rnd(T, Hkv, D), rnd(T, Hkv, D), table, torch.zeros_like(lengths), cu)
    bounds = torch.zeros((n, Hkv, 2, D), dtype=BF16, device=DEV)
    cache.bounds(table, torch.zeros_like(lengths), lengths, bounds)
    s = dict(cache=cache, table=table, lengths=lengths, bounds=bounds, k=rnd(B, Hkv, D), v=rnd(B, Hkv, D), q=rnd(B, Hq, D))
    s.update(o=torch.zeros_like(s["q"]), lse=torch.zeros((B, Hq), device=DEV),
             selected=torch.zeros((B, Hkv, 20), dtype=torch.int32, device=DEV), all=torch.zeros_like(s["q"]))
    return s


def step(s):
    starts = s["lengths"].clone()
    s["lengths"] += 1
    s["cache"].write(s["k"], s["v"], s["table"], starts)
    s["cache"].bounds(s["table"], starts, s["lengths"], s["bounds"])
    s["cache"].select(s["q"], s["bounds"], s["table"], s["lengths"], s["selected"])
    s["cache"].attend(s["q"], s["table"], s["lengths"], s["o"], s["lse"], s["selected"])
    s["cache"].attend(s["q"], s["table"], s["lengths"], s["all"])


@pytest.mark.parametrize("bits", [8, 4])
def test_graphs(bits):
    """A decode step captured twice, replayed in turn with eager work between: every replay is what the step is."""
    a, b = decode_state(bits=bits), decode_state(bits=bits)
    step(a), step(b)
    torch.cuda.synchronize()
    start = {k: x.clone() for k, x in b.items() if isinstance(x, torch.Tensor)}
    memory = b["cache"].memory.clone()
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(b)
    for k, x in start.items():
        b[k].copy_(x)
    b["cache"].memory.copy_(memory)
    for i in range(6):
        for s in (a, b):
            g = torch.Generator(device=DEV).manual_seed(i)
            for name in "qkv":
                s[name].copy_(torch.randn(s[name].shape, generator=g, device=DEV))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(a)
        torch.cuda.synchronize()
        for name in ("o", "lse", "selected", "all", "lengths", "bounds"):
            assert torch.equal(a[name], b[name]), (i, name)
        assert torch.equal(a["cache"].memory, b["cache"].memory)


def test_two_streams_at_once():
    """Calls on two caches from two streams, each with torch's workspaces of its own stream."""
    ss = [decode_state(seed=i, M=500) for i in range(2)]
    want = [decode_state(seed=i, M=500) for i in range(2)]
    for s in want:
        step(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ss]
    for s, st in zip(ss, streams):
        with torch.cuda.stream(st):
            step(s)
    torch.cuda.synchronize()
    for s, w in zip(ss, want):
        for name in ("o", "lse", "selected", "all", "bounds"):
            assert torch.equal(s[name], w[name])


@pytest.mark.parametrize("bits", [8, 4])
def test_binding_paths_agree(bits, monkeypatch):
    """The native argument path and the Python one make the same calls."""
    a, b = decode_state(bits=bits), decode_state(bits=bits)
    native = stepq.native()
    step(a)
    monkeypatch.setattr(stepq, "_native", stepq._PythonChecks)
    step(b)
    for name in ("o", "lse", "selected", "all", "lengths", "bounds"):
        assert torch.equal(a[name], b[name]), name
    for s in (a, b):
        s["back"] = [torch.zeros((5, 2, 64), device=DEV) for _ in range(2)]
        monkeypatch.setattr(stepq, "_native", native if s is a else stepq._PythonChecks)
        s["cache"].read(s["table"], s["lengths"] - 1, *s["back"])
        s["cache"].attend(s["q"], s["table"], s["lengths"], s["all"], scale=0.25)
    assert torch.equal(a["all"], b["all"]) and all(torch.equal(x, y) for x, y in zip(a["back"], b["back"]))


def example():
    spec = importlib.util.spec_from_file_location("shared_prefix", os.path.join(ROOT, "examples", "shared_prefix.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("P", [150, 160])
@pytest.mark.parametrize("bits,tol", [(8, 5e-2), (4, 0.5)])
def test_the_example_with_quantized_caches(bits, tol, P):
    """Against the same server with caches that are not quantized.  A held value is off by half a step of its row's
    (64 dimensions') largest magnitude, 1/254 or 1/14 of it: relative to the rows' norms that is 1/254 x sqrt(64) / (3
    sqrt(3)) or 18 times as much of 4 bits at most for a largest of 3 times the mean square; scores of up to a few units move by
    as much of them, values likewise.  One attention layer of the stack and the layer after it carry that on: 5 % and 50 %
    of the largest output.  All pages selected: the same outputs but for the order of sums."""
    m = example()
    outs = {}
    for name, kw in (("plain", {}), ("held", dict(cache_bits=bits)), ("all", dict(cache_bits=bits, select=40)),
                     ("few", dict(cache_bits=bits, select=4))):
        stack = m.Stack(kinds=("delta", "attention", "decay"), width=128, v_heads=4, qk_heads=2, d=64, q_heads=8, kv_heads=2,
                        head_dim=64, dtype=torch.float32)
        g = torch.Generator().manual_seed(3)
        draw = lambda n: torch.randn((n, stack.width), generator=g)
        prefix, prompts, more = draw(P), [draw(n) for n in (1, 70, 13)], [draw(3) for _ in range(3)]
        server = m.Server(stack, prefix.cuda(), 3, 80, page=16, quantized=False, **kw)
        outs[name] = [server.admit([p.cuda() for p in prompts])] + [server.step(x.cuda()) for x in more]
    size = torch.stack(outs["plain"]).abs().max()
    far = lambda a, b: float((torch.stack(outs[a]) - torch.stack(outs[b])).abs().max() / size)
    assert 1e-5 < far("held", "plain") <= tol, far("held", "plain")
    assert far("all", "held") <= 1e-4
    assert torch.isfinite(torch.stack(outs["few"])).all() and torch.equal(outs["few"][0], outs["held"][0])
