"""Decoding with the paged 4-bit cache: page tables, rotary positions, append, page selection and attention as a server runs them.

One attention layer with random weights stands for a model.  A few requests bring prompts of different lengths, which
go in as chunks; then every request decodes token by token, once over all that it holds and once over the pages that the
keys' boxes promise most for, and checks trees of drafted tokens, of which a path stays; one request ends on the way and its pages
serve another.

    python examples/kv_decode.py [--requests 8] [--prompt 4000] [--steps 64] [--pages 16] [--drafted 8]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2312_01712_amd import kv  # noqa: E402


class Layer:
    """Projections of one attention layer: x [T][width] to the rows of queries, keys and values, and back."""

    def __init__(self, width, heads, kv_heads, head_dim, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        new = lambda a, b: (torch.randn(a, b, device="cuda", generator=g) * a ** -0.5).bfloat16()
        self.qkv, self.out = new(width, (heads + 2 * kv_heads) * head_dim), new(heads * head_dim, width)

    def project(self, x):
        rows = (x @ self.qkv).unflatten(-1, (-1, self.head_dim))      # [T][heads + 2 kv_heads][head_dim]
        return rows[:, :self.heads], rows[:, self.heads:-self.kv_heads], rows[:, -self.kv_heads:]


class Server:
    def __init__(self, layer, requests, longest, n_pages):
        self.layer = layer
        self.cache = kv.KvCache(n_pages, layer.kv_heads, layer.head_dim)
        self.free_pages, self.free_state = self.cache.free_ring()
        self.lens = torch.zeros(requests, dtype=torch.int32, device="cuda")
        self.table = torch.full((requests, -(-longest // kv.PAGE)), -1, dtype=torch.int32, device="cuda")
        half = layer.head_dim // 2
        self.rotary = kv.Rotary([10000.0 ** (-i / half) for i in range(half)])

    def step(self, x, new, pages=0):
        """New tokens x [T][width] of all requests, `new` of each (a list; -1: the request ends); pages: how many pages a
        token looks at, 0 for all.  Returns the layer's output rows."""
        layer, cache = self.layer, self.cache
        q, k, v = layer.project(x)
        step = kv.plan(self.lens, torch.tensor(new, dtype=torch.int32, device="cuda"), self.table, self.free_pages,
                       self.free_state, max_tokens=x.shape[0])
        self.lens, self.free_state = step.kv_lens, step.free_state
        q, k = self.rotary(q, k, step.positions, out=(q, k))              # where they are, in the projection's rows
        cache.append(k, v, step.slots)
        selected = cache.select(q, step, pages) if pages else None
        out, _ = cache.attention(q, step, pages=selected, max_new=max(max(new), 1))
        return out.flatten(1) @ layer.out

    def check(self, x, parents, new, drafted, pick):
        """Trees of drafted tokens x [T][width], `new` of each request; parents, drafted [T]: the token of its request that each hangs on,
        and which it is.  pick: from the layer's output rows, the tokens that the model picks behind each.  Returns the
        output rows and those that stay (`kv.Kept`)."""
        layer, cache = self.layer, self.cache
        q, k, v = layer.project(x)
        step = kv.plan(self.lens, torch.tensor(new, dtype=torch.int32, device="cuda"), self.table, self.free_pages,
                       self.free_state, max_tokens=x.shape[0])
        tree = kv.tree(parents, step, max_nodes=max(max(new), 1))
        q, k = self.rotary(q, k, tree.positions, out=(q, k))
        cache.append(k, v, step.slots)
        out, _ = cache.tree_attention(q, step, tree)
        y = out.flatten(1) @ layer.out
        kept = kv.keep([cache], step, tree, drafted, pick(y), self.free_pages, step.free_state)
        self.lens, self.free_state = kept.lens, kept.free_state
        return y, kept


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=4000)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--pages", type=int, default=16)
    ap.add_argument("--drafted", type=int, default=8)
    a = ap.parse_args(argv)
    width, R = 1024, a.requests
    layer = Layer(width, heads=32, kv_heads=8, head_dim=128)
    prompts = [max(1, a.prompt * (i + 1) // R) for i in range(R)]
    longest = a.prompt + (2 + a.drafted) * a.steps + kv.PAGE
    server = Server(layer, R, longest, n_pages=R * -(-longest // kv.PAGE))
    for at in range(0, max(prompts), 1024):                           # prompts in chunks of 1024 tokens
        new = [min(1024, max(0, p - at)) for p in prompts]
        server.step(torch.randn(sum(new), width, device="cuda").bfloat16(), new)
    for pages in (0, a.pages):
        x = torch.randn(R, width, device="cuda").bfloat16()
        torch.cuda.synchronize()
        begin = time.perf_counter()
        for _ in range(a.steps):
            y = server.step(x, [1] * R, pages)
            x = y / y.float().std(-1, keepdim=True).bfloat16()        # the output is the next token's input
        torch.cuda.synchronize()
        took = (time.perf_counter() - begin) / a.steps
        print(f"{R} requests, {'all pages' if not pages else f'{pages} pages a token'}: {took * 1e6:.0f} us a step", flush=True)
    # trees of drafted tokens, each hanging on one of the three before it; the model's picks are random here, one of two tokens
    n = a.drafted
    parents = torch.tensor([max(i - 1 - i % 3, 0) if i else -1 for i in range(n)] * R, dtype=torch.int32, device="cuda")
    held = server.lens.clone()
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(a.steps):
        drafted = torch.randint(0, 2, (R * n,), dtype=torch.int32, device="cuda")
        server.check(torch.randn(R * n, width, device="cuda").bfloat16(), parents, [n] * R, drafted,
                     lambda y: (y[:, 0] > 0).int())
    torch.cuda.synchronize()
    took, stay = (time.perf_counter() - begin) / a.steps, (server.lens - held).sum().item() / a.steps / R
    assert bool((server.lens >= held + a.steps).all()) and int(server.free_state[2]) == 0
    print(f"{R} requests, {n} drafted tokens each: {took * 1e6:.0f} us a step, {stay:.1f} of them stay", flush=True)
    # the same tokens over all pages and over the selected ones
    x = torch.randn(R, width, device="cuda").bfloat16()
    lens, state = server.lens, server.free_state
    whole = server.step(x, [1] * R)
    server.lens, server.free_state = lens, state                      # the step again, from where it began
    part = server.step(x, [1] * R, a.pages)
    print(f"selected pages against all: {((whole - part).float().norm() / whole.float().norm()).item():.3f} of the output's norm")
    server.step(x[1:], [-1] + [1] * (R - 1))                          # the first request ends ...
    held = int(server.lens.sum())
    y = server.step(torch.randn(100 + R - 1, width, device="cuda").bfloat16(), [100] + [1] * (R - 1))  # ... and another starts
    assert int(server.lens.sum()) == held + 100 + R - 1 and int(server.free_state[2]) == 0 and bool(torch.isfinite(y).all())
    print(f"tokens held: {int(server.lens.sum())}, cache: {server.cache.pages.numel() / 2**20:.0f} MiB")
    return whole, part


if __name__ == "__main__":
    main()
