"""One attention layer of a server that drafts trees of tokens, end to end on the paged 4-bit cache.

Requests come with prompts of ragged lengths; every step a tree of tokens is
drafted for each of them, verified in one pass, and the accepted path stays:

* ``kv4_plan`` keeps the books on the GPU: pages of tokens that were not accepted go
  back, the next tokens get positions (a node's is its depth behind the context) and slots;
* prompts attend with ``window_prompt_attention`` (or ``prompt_attention``) to
  what ``kv4_read`` reads back of the cache;
* drafted tokens are appended with ``kv4_append`` and attend with
  ``tree_attention_kv4`` straight on the pages, each to the context and its ancestors;
* ``kv4_keep`` moves the accepted path together; the rest is dropped by the
  next step's plan;
* between steps a request may also decode one token with ``window_attention_kv4``.

Projections, the drafting and the choice of a path are stand-ins (random); the run
prints how far the last step's outputs are from attention over the read-back cache
in fp64.

    python examples/speculative_serving.py [--requests 16] [--steps 6] [--window 0]
"""
from __future__ import annotations

import argparse
import os
import random
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2405_16406_gb300 import spinq  # noqa: E402


class Layer:
    """The cache of one layer with its requests' lengths, page tables and free pages."""

    def __init__(self, requests, longest, heads=32, kv_heads=8, dim=128, page=64, base=500000.0, seed=0):
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        width = -(-longest // page)
        pages = requests * width
        self.cache = spinq.kv4_pages(pages, page, kv_heads, dim)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.lens, self.table = torch.zeros(requests, **i32), torch.full((requests, width), -1, **i32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.count = torch.full((1,), pages, **i32)
        theta = base ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * theta
        self.cos_sin = torch.stack((angle.cos(), angle.sin()), -1).float()

    def plan(self, add, total, drop=None, depths=None):
        return spinq.kv4_plan(self.lens, add, self.table, self.free, self.count, self.page, total, drop=drop, depths=depths)

    def append(self, fused, plan):
        """New tokens' projection output [T, (Hq + 2 Hkv) D] into the cache; the rotated queries."""
        hq, hk, d = self.heads, self.kv_heads, self.dim
        q, k, v = (t.unflatten(-1, (-1, d)) for t in fused.split((hq * d, hk * d, hk * d), -1))
        return spinq.kv4_append(q, k, v, self.cache, plan.slots, plan.positions, self.cos_sin)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def offsets(lens):
    return ints([0] + torch.tensor(lens).cumsum(0).tolist())


def draft(rng, nodes):
    """A tree: parents, and depths below the root."""
    parents = [-1] + [rng.randint(max(0, i - 6), i - 1) for i in range(1, nodes)]
    depths = []
    for p in parents:
        depths.append(0 if p < 0 else depths[p] + 1)
    return parents, depths


def choose(rng, parents):
    """An accepted path from the root down to a random node."""
    node, path = rng.randrange(len(parents)), []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def serve(requests=16, steps=6, heads=32, kv_heads=8, dim=128, page=64, longest_prompt=600, most_nodes=24, window=0, sinks=4,
          seed=0):
    """Prefill and verify; returns the last step's outputs and queries, its trees, and the layer before its paths are kept."""
    rng = random.Random(seed)
    layer = Layer(requests, longest_prompt + (steps + 1) * most_nodes, heads, kv_heads, dim, page, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    project = lambda n: torch.randn((n, (heads + 2 * kv_heads) * dim), generator=g, device="cuda").half()   # noqa: E731

    # the prompts, packed
    lens = [rng.randint(1, longest_prompt) for _ in range(requests)]
    total = sum(lens)
    plan = layer.plan(ints(lens), total)
    q = layer.append(project(total), plan)
    k, v = spinq.kv4_read(layer.cache, layer.table, plan.cu_tokens, total)
    if window:
        spinq.window_prompt_attention(q, k, v, plan.cu_tokens, plan.cu_tokens, max(lens), max(lens), window, sinks)
    else:
        spinq.prompt_attention(q, k, v, plan.cu_tokens, plan.cu_tokens, max(lens), max(lens))

    drop = None
    for step in range(steps):
        trees = [draft(rng, rng.randint(1, most_nodes)) for _ in range(requests)]
        nodes = [len(p) for p, _ in trees]
        total, most = sum(nodes), max(nodes)
        plan = layer.plan(ints(nodes), total, drop=drop, depths=ints([d for _, t in trees for d in t]))
        q = layer.append(project(total), plan)
        parents = ints([x for p, _ in trees for x in p])
        out = spinq.tree_attention_kv4(q, layer.cache, layer.table, layer.lens, plan.cu_tokens, most, parents, window, sinks)
        if step == steps - 1:
            return out, q, trees, layer, plan
        paths = [choose(rng, p) for p, _ in trees]
        deepest = max(map(len, paths))
        # (a request that got no pages has no drafted tokens: nothing of it is kept or dropped)
        spinq.kv4_keep(layer.cache, layer.table, layer.lens - ints(nodes), ints([p + [0] * (deepest - len(p)) for p in paths]),
                       ints([len(p) for p in paths]) * plan.granted)
        drop = ints([n - len(p) for n, p in zip(nodes, paths)]) * plan.granted
        if step % 2:   # a step without a draft: the last tokens' queries again, one each
            last = (plan.cu_tokens[1:] - 1).long()
            layer.plan(None, 0, drop=drop)
            drop = None
            spinq.window_attention_kv4(q[last], layer.cache, layer.table, layer.lens, window, sinks)


def attention_over_read_back(q, trees, layer, plan, window, sinks):
    """The last step in fp64 over the read-back cache."""
    lens = layer.lens.tolist()
    cu = offsets(lens)
    k, v = (x.double() for x in spinq.kv4_read(layer.cache, layer.table, cu, sum(lens)))
    group, out, at = layer.heads // layer.kv_heads, [], 0
    for b, (parents, depths) in enumerate(trees):
        n, first = len(parents), lens[b] - len(parents)
        kb, vb = k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]]
        place = torch.tensor(list(range(first)) + [first + d for d in depths])
        lines = []
        for p in parents:
            lines.append((lines[p] if p >= 0 else []) + [len(lines)])
        seen = torch.zeros((n, lens[b]), dtype=torch.bool)
        seen[:, :first] = True
        for i, line in enumerate(lines):
            seen[i, [first + x for x in line]] = True
        if window:
            here = first + torch.tensor(depths)[:, None]
            seen &= (here - place < window) | (place < sinks)
        x = q[at:at + n].double().view(n, layer.kv_heads, group, -1)
        w = torch.einsum("nhgd,thd->nhgt", x, kb) / layer.dim ** 0.5
        w = torch.softmax(w.masked_fill(~seen.cuda()[:, None, None], -torch.inf), -1)
        out.append(torch.einsum("nhgt,thd->nhgd", w, vb).flatten(1, 2))
        at += n
    return torch.cat(out)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--window", type=int, default=0)
    a = ap.parse_args()
    serve(a.requests, 1, window=a.window)   # loads the kernels
    torch.cuda.synchronize()
    t = time.perf_counter()
    out, q, trees, layer, plan = serve(a.requests, a.steps, window=a.window)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    ref = attention_over_read_back(q, trees, layer, plan, a.window, 4)
    rel = float((out.double() - ref).norm() / ref.norm())
    print(f"{a.requests} requests, {a.steps} drafted steps: {t * 1e3:.1f} ms; last step against fp64 over the read-back "
          f"cache: {rel:.2e}")


if __name__ == "__main__":
    main()
