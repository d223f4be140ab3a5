"""One attention layer served from the paged 4-bit cache, end to end.

A batch of requests shares an instruction text.  The text is prefilled once;
each request's own prompt then arrives in one packed batch of ragged lengths,
and every request decodes a few tokens:

* every new token goes through ``kv4_append`` (norms of the query and key heads,
  RoPE, R3, the 4-bit quantizer, the pages);
* a prompt attends with ``prompt_attention`` to what ``kv4_read`` reads back of
  the cache, its context included, so that prefill and decode see the same keys;
* a decode step attends with ``prefix_attention_kv4`` straight on the pages, the
  shared text computed once for the whole batch.

Projections and the rest of a model are stand-ins (random queries, keys and
values); the run prints how far the decode outputs are from attention over the
read-back cache in fp64.

    python examples/paged_serving.py [--requests 16] [--shared 2000] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2405_16406_gb300 import spinq  # noqa: E402


class PagedLayer:
    """The cache of one layer, its pages handed out in order, and its norms and rotation table."""

    def __init__(self, heads=32, kv_heads=8, dim=128, pages=4096, page=64, max_pos=1 << 16, base=500000.0, seed=0):
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.cache = spinq.kv4_pages(pages, page, kv_heads, dim)
        self.free = 0
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.q_weight, self.k_weight = ((1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).half() for _ in range(2))
        theta = base ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
        angle = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * theta
        self.cos_sin = torch.stack((angle.cos(), angle.sin()), -1).float()

    def new_pages(self, n):
        self.free += n
        assert self.free <= self.cache.k_codes.shape[0], "the cache is full"
        return torch.arange(self.free - n, self.free, dtype=torch.int32, device="cuda")

    def append(self, fused, slots, positions):
        """New tokens' projection output [T, (Hq + 2 Hkv) D] into the cache; the rotated queries."""
        hq, hk, d = self.heads, self.kv_heads, self.dim
        q, k, v = (t.unflatten(-1, (-1, d)) for t in fused.split((hq * d, hk * d, hk * d), -1))
        return spinq.kv4_append(q, k, v, self.cache, slots, positions, self.cos_sin, self.q_weight, self.k_weight)


def offsets(lens):
    return torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def serve(requests=16, shared=2000, steps=8, heads=32, kv_heads=8, dim=128, page=64, seed=0):
    """Prefill and decode; returns the decode outputs [steps, requests, heads, dim], the last
    step's rotated queries, the layer, and the tables and lengths of its sequences."""
    layer = PagedLayer(heads, kv_heads, dim, pages=(shared + requests * 400) // page + 2 * requests + 2, page=page,
                       seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    width = (heads + 2 * kv_heads) * dim
    project = lambda n: torch.randn((n, width), generator=g, device="cuda").half()   # noqa: E731

    # the instruction text: appended, read back, attended to
    text = layer.new_pages(-(-shared // page))
    at = torch.arange(shared, device="cuda")
    q = layer.append(project(shared), text.long()[at // page] * page + at % page, at.int())
    cu = offsets([shared])
    k, v = spinq.kv4_read(layer.cache, text[None], cu, shared)
    spinq.prompt_attention(q, k, v, cu, cu, shared, shared)

    # the requests' own prompts, packed; their context is the text
    lens = torch.randint(1, 300, (requests,), generator=torch.Generator().manual_seed(seed)).tolist()
    most = max(lens) + steps
    tables = torch.stack([layer.new_pages(-(-most // page)) for _ in range(requests)])
    row = torch.repeat_interleave(torch.arange(requests, device="cuda"), torch.tensor(lens, device="cuda"))
    cu = offsets(lens)
    own = torch.arange(sum(lens), device="cuda") - cu.long()[row]
    q = layer.append(project(sum(lens)), tables.long()[row, own // page] * page + own % page, (own + shared).int())
    # a request's keys: the text's tokens, then its own, each read into place
    keys = offsets([shared + n for n in lens])
    k = torch.empty((int(keys[-1]), kv_heads, dim), dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    whole = offsets([shared])
    for b, a in enumerate(keys.tolist()[:-1]):
        m, e = a + shared, a + shared + lens[b]
        spinq.kv4_read(layer.cache, text[None], whole, shared, k=k[a:m], v=v[a:m])
        spinq.kv4_read(layer.cache, tables[b:b + 1], offsets(lens[b:b + 1]), lens[b], k=k[m:e], v=v[m:e])
    spinq.prompt_attention(q, k, v, cu, keys, max(lens), shared + max(lens))

    # decode: a token per request and step
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    each = torch.arange(requests, device="cuda")
    outs = []
    for _ in range(steps):
        t = length.long()
        q = layer.append(project(requests), tables.long()[each, t // page] * page + t % page, length + shared)
        length += 1
        outs.append(spinq.prefix_attention_kv4(q, layer.cache, text, shared, tables, length))
    return torch.stack(outs), q, layer, text, tables, length


def attention_over_read_back(q, layer, text, shared, tables, length):
    """The last decode step in fp64 over the read-back cache."""
    kt, vt = spinq.kv4_read(layer.cache, text[None], offsets([shared]), shared)
    lens = length.tolist()
    cu = offsets(lens)
    ko, vo = spinq.kv4_read(layer.cache, tables, cu, sum(lens))
    group, out = layer.heads // layer.kv_heads, []
    for b, (a, e) in enumerate(zip(cu.tolist()[:-1], cu.tolist()[1:])):
        k, v = torch.cat((kt, ko[a:e])).double(), torch.cat((vt, vo[a:e])).double()
        x = q[b].double().view(layer.kv_heads, group, -1)
        w = torch.softmax(torch.einsum("hgd,thd->hgt", x, k) / layer.dim ** 0.5, -1)
        out.append(torch.einsum("hgt,thd->hgd", w, v).flatten(0, 1))
    return torch.stack(out)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--shared", type=int, default=2000)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    serve(a.requests, a.shared, 1)   # loads the kernels
    torch.cuda.synchronize()
    t = time.perf_counter()
    outs, q, layer, text, tables, length = serve(a.requests, a.shared, a.steps)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    ref = attention_over_read_back(q, layer, text, a.shared, tables, length)
    rel = float((outs[-1].double() - ref).norm() / ref.norm())
    print(f"{a.requests} requests behind {a.shared} shared tokens, {a.steps} decode steps: {t * 1e3:.1f} ms; "
          f"last step against fp64 over the read-back cache: {rel:.2e}")


if __name__ == "__main__":
    main()
