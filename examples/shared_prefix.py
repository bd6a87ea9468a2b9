"""Serve requests that share a long prefix on a small hybrid stack.

The stack has three kinds of layers, with random weights: "delta" (a gated
Delta rule, its states quantized in a pool), "decay" (linear attention with a
decay per head, fp32 states) and "attention" (softmax over paged caches).
- The prefix goes through once: one state per recurrent layer, one set of pages
  per attention layer.
- Each request's own prompt starts from that state (stepq_prompt with in_ids all
  0) and reads those pages (stepq_prefix_attention, a row per prompt token).
- The delta layers' states are fitted and packed into pools.
- Decoding: Pool.step, stepq_state_step and stepq_prefix_attention, one token of
  every request at a time.

    python examples/shared_prefix.py --requests 64 --prefix 4096
"""
import argparse
import os
import sys
import time
from dataclasses import dataclass

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38169_amd import stepq  # noqa: E402


@dataclass
class Stack:
    """Sizes and weights of the layers; a token is a vector of `width`."""
    kinds: tuple = ("delta", "delta", "decay", "attention")
    width: int = 1024
    v_heads: int = 16
    qk_heads: int = 4
    d: int = 128                # of the recurrent heads
    q_heads: int = 16
    kv_heads: int = 2
    head_dim: int = 128
    dtype: torch.dtype = torch.bfloat16
    device: str = "cuda"
    seed: int = 0

    def __post_init__(self):
        g = torch.Generator().manual_seed(self.seed)
        draw = lambda n, m: (torch.randn((n, m), generator=g) * n ** -0.5).to(self.dtype).to(self.device)
        self.w_in = [draw(self.width, sum(self.widths(k))) for k in self.kinds]
        self.w_out = [draw(self.widths(k)[-1], self.width) for k in self.kinds]
        self.w_gate = [draw(self.width, 2 * self.v_heads) for _ in self.kinds]

    def widths(self, kind):
        if kind == "attention":
            return self.q_heads * self.head_dim, self.kv_heads * self.head_dim, self.kv_heads * self.head_dim, \
                self.q_heads * self.head_dim
        return self.qk_heads * self.d, self.qk_heads * self.d, self.v_heads * self.d, self.v_heads * self.d

    def project(self, i, x):
        """The layer's q, k, v of tokens x [n][width], and alpha, beta of a recurrent layer: [n][heads][d], [n][heads]."""
        kind, n = self.kinds[i], x.shape[0]
        y = x * torch.rsqrt((x.float() ** 2).mean(-1, keepdim=True) + 1e-6).to(x.dtype)
        q, k, v = (y @ self.w_in[i]).split(self.widths(kind), -1)[:3]
        if kind == "attention":
            return tuple(z.reshape(n, -1, self.head_dim) for z in (q, k, v)) + (None, None)
        q, k, v = (z.reshape(n, -1, self.d) for z in (q, k, v))
        q, k = (z / z.float().norm(dim=-1, keepdim=True).clamp_min(1e-6).to(z.dtype) for z in (q, k))
        a, b = (y @ self.w_gate[i]).split(self.v_heads, -1)
        return q, k, v, torch.sigmoid(a + 4), torch.sigmoid(b)

    def add(self, i, x, o):
        return x + o.reshape(x.shape[0], -1).to(x.dtype) @ self.w_out[i]


class Server:
    """States and caches of up to `capacity` requests over one prefix [P][width]."""

    def __init__(self, stack: Stack, prefix, capacity: int, own_tokens: int, page: int = 64, quantized: bool = True):
        s = self.stack = stack
        self.page, self.P, self.capacity, self.quantized = page, prefix.shape[0], capacity, quantized
        self.own_pages = -(-own_tokens // page)
        n_prefix = -(-self.P // page)
        i32 = dict(dtype=torch.int32, device=s.device)
        self.prefix_pages = torch.arange(n_prefix, **i32)
        self.table = n_prefix + torch.arange(capacity * self.own_pages, **i32).view(capacity, -1)
        self.ids = torch.arange(capacity, **i32)
        self.lengths = torch.zeros(capacity, **i32)
        self.pools, self.states, self.start, self.caches = {}, {}, {}, {}
        for i, kind in enumerate(s.kinds):
            if kind == "attention":
                n = n_prefix + capacity * self.own_pages
                self.caches[i] = [torch.zeros((n, s.kv_heads, page, s.head_dim), dtype=s.dtype, device=s.device) for _ in "kv"]
            else:
                self.states[i] = torch.zeros((capacity, s.v_heads, s.d, s.d), device=s.device)
                if kind == "delta" and quantized:
                    bits = np.full((s.v_heads, s.d), 8, np.uint8)
                    self.pools[i] = stepq.Pool(capacity, s.v_heads, s.qk_heads, s.d, s.d, bits)
        self._prefix(prefix)

    def _write(self, i, table, at, k, v):
        """Rows of the caches of the tokens at positions `at` of their pages."""
        pages = table.gather(-1, (at // self.page).long().unsqueeze(-1)).squeeze(-1).long()
        for cache, x in zip(self.caches[i], (k, v)):
            cache[pages, :, (at % self.page).long()] = x

    def _attend(self, i, q, prefix_len, table, lengths):
        o = torch.empty_like(q)
        stepq.stepq_prefix_attention(q.contiguous(), *self.caches[i], self.prefix_pages, prefix_len, table, lengths, o)
        return o

    def _prefix(self, x):
        s, P = self.stack, self.P
        at = torch.arange(P, dtype=torch.int32, device=s.device)
        table = self.prefix_pages.expand(P, -1).contiguous()       # every token reads the pages up to itself
        for i, kind in enumerate(s.kinds):
            q, k, v, alpha, beta = s.project(i, x)
            if kind == "attention":
                self._write(i, table, at, k, v)
                o = self._attend(i, q, 0, table, at + 1)
            else:
                o = torch.empty_like(v, memory_format=torch.contiguous_format)
                self.start[i] = torch.empty((1, s.v_heads, s.d, s.d), device=s.device)
                stepq.stepq_prompt(q, k, v, alpha, beta, o, self.start[i], rule=_rule(kind))
            x = s.add(i, x, o)
        return x

    def admit(self, prompts):
        """The requests' own prompts [T_b][width], one per request of the capacity; returns each one's last output."""
        s, B = self.stack, self.capacity
        n = [p.shape[0] for p in prompts]
        if len(n) != B or min(n) < 1 or max(n) > self.own_pages * self.page:
            raise ValueError("a prompt of 1 token or more, within its pages, for each request")
        cu = torch.tensor([0] + n, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(s.device)
        self.lengths.copy_(torch.tensor(n, dtype=torch.int32))
        owner = torch.repeat_interleave(torch.arange(B, device=s.device), self.lengths.long())
        at = torch.arange(len(owner), dtype=torch.int32, device=s.device) - cu[owner]
        table, from_prefix = self.table[owner], torch.zeros(B, dtype=torch.int32, device=s.device)
        x = torch.cat(list(prompts))
        for i, kind in enumerate(s.kinds):
            q, k, v, alpha, beta = s.project(i, x)
            if kind == "attention":
                self._write(i, table, at, k, v)
                o = self._attend(i, q, self.P, table, at + 1)
            else:
                o = torch.empty_like(v, memory_format=torch.contiguous_format)
                stepq.stepq_prompt(q, k, v, alpha, beta, o, self.states[i], rule=_rule(kind), cu_seqlens=cu,
                                   state_in=self.start[i], in_ids=from_prefix)
                if i in self.pools:
                    r, c = stepq.stepq_setup_fit(self.states[i].cpu())
                    self.pools[i].load(self.ids, self.states[i], torch.from_numpy(r).to(s.device),
                                       torch.from_numpy(c).to(s.device))
            x = s.add(i, x, o)
        return x[cu[1:].long() - 1]

    def step(self, x):
        """One token of every request: [B][width] in and out."""
        s, B = self.stack, self.capacity
        at = self.lengths.clone()
        self.lengths += 1
        for i, kind in enumerate(s.kinds):
            q, k, v, alpha, beta = s.project(i, x)
            if kind == "attention":
                self._write(i, self.table, at, k, v)
                o = self._attend(i, q, self.P, self.table, self.lengths)
            else:
                o = torch.empty((B, s.v_heads, s.d), device=s.device)
                args = tuple(z.contiguous() for z in (q, k, v, alpha, beta))
                if i in self.pools:
                    self.pools[i].step(self.ids, *args, o)
                else:
                    stepq.stepq_state_step(self.states[i], self.ids, *args, o, rule=_rule(kind))
            x = s.add(i, x, o)
        return x


def _rule(kind):
    return stepq.STEPQ_RULE_DELTA if kind == "delta" else stepq.STEPQ_RULE_DECAY


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--requests", type=int, default=64)
    p.add_argument("--prefix", type=int, default=4096)
    p.add_argument("--prompt", type=int, default=200, help="longest prompt of a request's own")
    p.add_argument("--steps", type=int, default=32)
    a = p.parse_args()
    stack = Stack()
    g = torch.Generator().manual_seed(1)
    draw = lambda n: torch.randn((n, stack.width), generator=g).to(stack.dtype).to(stack.device)
    prefix, prompts = draw(a.prefix), [draw(n) for n in torch.randint(1, a.prompt + 1, (a.requests,), generator=g).tolist()]

    def timed(what, f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        y = f()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - t) * 1e3:.2f} ms", flush=True)
        return y

    for _ in range(2):                          # the second time without first-use costs
        server = timed(f"prefix of {a.prefix} tokens", lambda: Server(stack, prefix, a.requests, a.prompt + 2 * a.steps))
        x = timed(f"{sum(map(len, prompts))} tokens of {a.requests} prompts, states packed", lambda: server.admit(prompts))

    def decode(n):
        y = x
        for _ in range(n):
            y = server.step(y / y.float().square().mean(-1, keepdim=True).sqrt().to(y.dtype))
        return y

    decode(a.steps)
    y = timed(f"{a.steps} steps of {a.requests} requests", lambda: decode(a.steps))
    if not torch.isfinite(y).all():
        raise SystemExit("outputs that are not finite")


if __name__ == "__main__":
    main()
