"""Operators for speculative decoding and sliding windows on the paged 4-bit
cache: the cases they are measured on, and their plain form.

* ``plan``: the step's bookkeeping from the lengths of the requests: pages of
  dropped tokens go back to the free list, pages of new tokens come from it,
  and every new token gets its position and its slot (``spinq.kv4_plan``).
* ``keep``: the accepted path of every drafted tree moves together in the cache
  (``spinq.kv4_keep``).
* ``prompt``: attention over packed ragged prompts with grouped heads where a
  query sees the last ``window`` positions and the first ``sinks`` tokens
  (``spinq.window_prompt_attention``).
* ``decode``: one query per sequence and head over the last ``window`` tokens and
  the first ``sinks`` of its 4-bit pages (``spinq.window_attention_kv4``).
* ``tree``: the drafted tokens of every sequence, a tree given by its parents,
  over the sequence's context and their own ancestors, straight on the 4-bit
  pages (``spinq.tree_attention_kv4``).

``own`` false computes them in elementary torch operations in 32 bits, rounded
once at the end; ``own`` true calls the library.  Lengths, trees and paths of a case
come from its own numbers (``lens_seed``), everything else from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False


# ------------------------------------------------------------------ the cases
def listed():
    heads = {"heads": 32, "kv_heads": 8, "head_dim": 128}
    return [
        # one decode step of eight requests: the call's latency counts
        {"name": "plan 8 x 1", "op": "plan", "batch": 8, "shortest": 1, "longest": 1, "context": 4096, "page": 64,
         "padding": 0, "scarce": False, "lens_seed": 0},
        # a full server takes new prompts in place of old ones, and runs out of pages for the last of them
        {"name": "plan 1000 ragged prompts", "op": "plan", "batch": 1000, "shortest": 1, "longest": 509, "context": 0,
         "page": 16, "padding": 1000, "scarce": True, "lens_seed": 1},
        # four requests keep a few accepted tokens of a step
        {"name": "keep 4 x 3", "op": "keep", "batch": 4, "context": 500, "nodes": 16, "path": 4, "kv_heads": 8,
         "head_dim": 128, "page": 64, "lens_seed": 2},
        # a large batch of deep trees
        {"name": "keep 256 x 11", "op": "keep", "batch": 256, "context": 333, "nodes": 64, "path": 12, "kv_heads": 8,
         "head_dim": 128, "page": 16, "lens_seed": 3},
        # a few short prompts with small heads
        {"name": "prompt few short", "op": "prompt", "batch": 3, "shortest": 1, "longest": 61, "context": 0, "window": 16,
         "sinks": 4, "heads": 8, "kv_heads": 2, "head_dim": 64, "lens_seed": 4},
        # packed prompts of many lengths, a narrow window
        {"name": "prompt ragged, window 512", "op": "prompt", "batch": 16, "shortest": 1, "longest": 4001, "context": 0,
         "window": 512, "sinks": 4, **heads, "lens_seed": 5},
        # whole long prompts
        {"name": "prompt 2 x 16384, window 4096", "op": "prompt", "batch": 2, "shortest": 16384, "longest": 16384,
         "context": 0, "window": 4096, "sinks": 64, **heads, "lens_seed": 0},
        # one sequence decodes: latency counts
        {"name": "decode 1 x 1024", "op": "decode", "batch": 1, "shortest": 5001, "longest": 5001, "window": 1024,
         "sinks": 4, **heads, "page": 64, "lens_seed": 0},
        # a serving batch of long sequences with a usual window
        {"name": "decode 128 x 4096", "op": "decode", "batch": 128, "shortest": 700, "longest": 30011, "window": 4096,
         "sinks": 4, **heads, "page": 64, "lens_seed": 6},
        # one sequence verifies a small tree: latency counts
        {"name": "tree 1 x 8 nodes", "op": "tree", "batch": 1, "least": 8, "nodes": 8, "shortest": 1000, "longest": 1000,
         "window": 0, "sinks": 0, **heads, "page": 64, "lens_seed": 7},
        # ragged contexts and trees with small heads and a window
        {"name": "tree 24 ragged, window 1000", "op": "tree", "batch": 24, "least": 1, "nodes": 25, "shortest": 0,
         "longest": 6007, "window": 1000, "sinks": 5, "heads": 8, "kv_heads": 8, "head_dim": 64, "page": 16, "lens_seed": 8},
        # a serving batch verifies large trees over long contexts
        {"name": "tree 32 x 64 nodes", "op": "tree", "batch": 32, "least": 64, "nodes": 64, "shortest": 9001,
         "longest": 16384, "window": 0, "sinks": 0, **heads, "page": 64, "lens_seed": 9},
    ]


def _spread(rng, low, high):
    """A whole number from low to high, spread over the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(("plan", "keep", "prompt", "prompt", "decode", "decode", "tree", "tree", "tree"))
    heads, kv_heads, dim = rng.choice(((32, 8, 128), (28, 4, 128), (8, 8, 64), (16, 2, 64), (20, 4, 128),
                                       (32, 8, 64), (8, 1, 128)))
    page = rng.choice((16, 32, 64, 128, 256))
    case = {"op": op, "lens_seed": rng.randrange(1 << 20)}
    if op == "plan":
        longest = _spread(rng, 1, 509)
        case.update(batch=_spread(rng, 1, 1000), longest=longest, shortest=_spread(rng, 1, longest),
                    context=rng.choice((0, _spread(rng, 1, 5000))), page=page,
                    padding=rng.choice((0, _spread(rng, 1, 1000))), scarce=rng.random() < 0.3)
        return case
    case.update(kv_heads=kv_heads, head_dim=dim)
    if op == "keep":
        path = _spread(rng, 1, 12)
        case.update(batch=_spread(rng, 1, 256), context=_spread(rng, 1, 333), nodes=path + _spread(rng, 4, 52), path=path,
                    page=page)
        return case
    window, sinks = _spread(rng, 1, 4096), rng.choice((0, 1, 4, 4, 64, 200))
    case.update(heads=heads, window=window, sinks=sinks)
    if op == "prompt":
        longest = _spread(rng, 1, 16384)
        context = rng.choice((0, 0, _spread(rng, 1, 4096)))
        # no more pairs of a query and a key than the largest listed case has
        most = max(1, min(16, int(2 * 16384 * 4096 * 32 / (longest * min(window + sinks, longest + context) * heads))))
        case.update(batch=_spread(rng, 1, most), longest=longest, shortest=_spread(rng, 1, longest), context=context)
    elif op == "decode":
        longest = _spread(rng, 1, 30011)
        case.update(batch=_spread(rng, 1, 128), longest=longest, shortest=rng.choice((0, _spread(rng, 1, longest))), page=page,
                    window=rng.choice((window, window, 0 if longest <= 4096 else window)))
    else:
        longest = _spread(rng, 1, 16384)
        nodes = _spread(rng, 1, 128)
        most = max(1, min(32, int(32 * 64 * 12000 * 32 / (nodes * longest * heads))))
        case.update(batch=_spread(rng, 1, most), longest=longest, shortest=rng.choice((0, _spread(rng, 1, longest))),
                    nodes=nodes, least=_spread(rng, 1, nodes), page=page,
                    window=rng.choice((0, 0, window)))
    return case


def _lengths(case):
    r = random.Random(case["lens_seed"])
    return [r.randint(case["shortest"], case["longest"]) for _ in range(case["batch"])]


def _trees(case):
    """Each sequence's tree as the parents of its nodes: a node's parent comes before it, the first is the root."""
    r = random.Random(case["lens_seed"] + 1)
    return [[-1] + [r.randint(max(0, i - 9), i - 1) for i in range(1, r.randint(case["least"], case["nodes"]))]
            for _ in range(case["batch"])]


def _paths(case):
    """Accepted nodes of each sequence's tree, stored level by level: the first is the root, the others lie
    behind the first ``path`` nodes."""
    r = random.Random(case["lens_seed"] + 2)
    return [[0] + sorted(r.sample(range(case["path"], case["nodes"]), r.randint(0, min(case["path"] - 1, case["nodes"] - case["path"]))))
            for _ in range(case["batch"])]


# ----------------------------------------------------------------- the inputs
def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _pages_of(gen, lens, page, first=None, sinks=0):
    """Page tables of sequences of the given lengths, pages in random order, and the number of pages.  Pages that lie
    before token ``first`` of their sequence and behind its ``sinks`` have been given back: -1."""
    width = max(1, max((n + page - 1) // page for n in lens))
    at = torch.arange(width, device="cuda")[None]
    have = at < ((_ints(lens, torch.int64) + page - 1) // page)[:, None]
    if first is not None:
        have &= (at >= (_ints(first, torch.int64) // page)[:, None]) | (at * page < sinks)
    total = max(1, int(have.sum()))
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    table[have] = order[:int(have.sum())]
    return table, total


def _random_pages(gen, pages, case):
    """Pages as the quantizer leaves them: codes spread like a normal row's, scales of rows of unit variance."""
    shape = (pages, case["kv_heads"], case["page"], case["head_dim"] // 2)

    def codes():
        out = torch.empty(shape, dtype=torch.uint8, device="cuda")
        for at in range(0, pages, 512):   # a part at a time: the normal draws are 16 times the codes
            part = (min(512, pages - at),) + shape[1:]
            low = (torch.randn(part, generator=gen, device="cuda") * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            high = (torch.randn(part, generator=gen, device="cuda") * 2.7 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            out[at:at + 512] = low | (high << 4)
        return out

    scales = torch.empty((pages, case["kv_heads"], case["page"], 4), device="cuda")
    for at in (0, 2):
        step = 0.36 * (1 + 0.1 * torch.randn(shape[:3], generator=gen, device="cuda")).clamp_(0.5, 2)
        scales[..., at] = step
        scales[..., at + 1] = -7.5 * step + 0.1 * torch.randn(shape[:3], generator=gen, device="cuda")
    return codes(), codes(), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).half()

    s = dict(case)
    dim, hk, hq = case.get("head_dim"), case.get("kv_heads"), case.get("heads")
    if case["op"] == "plan":
        # a step drops the last tokens of every sequence and adds as many as the step before did: the state is the same
        # after every step.  Where pages are scarce the last sequences got none in the step before either.
        page, add = case["page"], _lengths(case)
        start = [case["context"]] * len(add)
        want = [(a + n + page - 1) // page - (a + page - 1) // page for a, n in zip(start, add)]
        short = sum(want) * 4 // 5 if case["scarce"] else sum(want)
        gets, left = [], short
        for n in want:
            gets.append(n == 0 or (n <= left and len(gets) == sum(gets)))
            left -= n if gets[-1] else 0
        lens = [a + n if g else a for a, n, g in zip(start, add, gets)]
        held = [(n + page - 1) // page for n in lens]
        spare = left if case["scarce"] else left + 100
        pages = sum(held) + spare
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        width = max(1, max((a + n + page - 1) // page for a, n in zip(start, add)))
        s["table"] = torch.full((len(add), width), -1, dtype=torch.int32, device="cuda")
        have = torch.arange(width, device="cuda")[None] < _ints(held, torch.int64)[:, None]
        s["table"][have] = order[spare:]
        s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        s["free"][:spare] = order[:spare]
        s["count"] = _ints([spare])
        s["lens"], s["add"] = _ints(lens), _ints(add)
        # a sequence that ends may be dropped by any number from its length on
        s["dropped"] = _ints([n - a if case["context"] else 1 << 20 for n, a in zip(lens, start)])
        s["total"] = sum(add) + case["padding"]
    elif case["op"] == "keep":
        ends = [case["context"] + case["nodes"]] * case["batch"]
        s["table"], pages = _pages_of(gen, ends, case["page"])
        s["k_codes"], s["v_codes"], s["scales"] = _random_pages(gen, pages, case)
        s["starts"] = _ints([case["context"]] * case["batch"])
        paths = _paths(case)
        s["accepted"] = _ints([p + [0] * (case["path"] - len(p)) for p in paths])
        s["counts"] = _ints([len(p) for p in paths])
    elif case["op"] == "prompt":
        lens = _lengths(case)
        total = sum(lens)
        keys = [n + case["context"] for n in lens]
        fused = normal(total, (hq + 2 * hk) * dim)   # strided rows, as the projection leaves them
        s["q"] = fused[:, :hq * dim].view(total, hq, dim)
        s["q"].mul_(2)
        if case["context"]:
            s["k"], s["v"] = normal(sum(keys), hk, dim), normal(sum(keys), hk, dim)
        else:
            s["k"] = fused[:, hq * dim:(hq + hk) * dim].view(total, hk, dim)
            s["v"] = fused[:, (hq + hk) * dim:].view(total, hk, dim)
        s["cu_q"], s["cu_k"] = _ints(_offsets(lens)), _ints(_offsets(keys))
        s["max_q"], s["max_k"] = max(lens), max(keys)
    elif case["op"] == "decode":
        lens = _lengths(case)
        first = [max(0, n - case["window"]) if case["window"] else 0 for n in lens]
        s["table"], pages = _pages_of(gen, lens, case["page"], first, case["sinks"])
        s["k_codes"], s["v_codes"], s["scales"] = _random_pages(gen, pages, case)
        s["lens"] = _ints(lens)
        s["most"] = max(lens)
        s["q"] = normal(case["batch"], hq, dim, scale=2.0)
    else:
        trees = _trees(case)
        lens = [n + len(t) for n, t in zip(_lengths(case), trees)]
        first = [max(0, n - len(t) - case["window"]) if case["window"] else 0 for n, t in zip(lens, trees)]
        s["table"], pages = _pages_of(gen, lens, case["page"], first, case["sinks"])
        s["k_codes"], s["v_codes"], s["scales"] = _random_pages(gen, pages, case)
        s["lens"] = _ints(lens)
        s["most"] = max(lens)
        s["parents"] = _ints([p for t in trees for p in t])
        s["cu_q"] = _ints(_offsets([len(t) for t in trees]))
        s["max_q"] = max(len(t) for t in trees)
        s["q"] = normal(len(s["parents"]), hq, dim, scale=2.0)
    return s


# ------------------------------------------------------------- the plain form
def _expanded(s, table, token, which):
    """Values [..., Hkv, D] of the tokens at positions `token` [B, n] of the page tables `table` [B, W]."""
    page, slot = token // s["page"], token % s["page"]
    at = table.long().gather(-1, page).clamp(min=0)
    packed = s["k_codes" if which == 0 else "v_codes"][at, :, slot]
    scale = s["scales"][at, :, slot]
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).float()
    return code * scale[..., 2 * which, None] + scale[..., 2 * which + 1, None]


def _softmax_product(scores, seen, v):
    """softmax(scores where seen) v; a row without a visible key gives zeros."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    weight = torch.exp(scores - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = weight.sum(-1, keepdim=True)
    return torch.where(total > 0, torch.matmul(weight, v) / total, torch.zeros_like(total))


def _plain_plan(s):
    page, total, table = s["page"], s["total"], s["table"]
    lens, add = s["lens"].long(), s["add"].long()
    capacity, count = table.shape[1] * page, s["count"].long()
    pages = lambda n: (n + page - 1) // page   # noqa: E731
    start = (lens - s["dropped"].long()).clamp(min=0)
    kept, freed = pages(start), pages(lens) - pages(start)
    ends = torch.cumsum(add, 0)
    fits = (add == 0) | ((ends <= total) & (start + add <= capacity))
    need = torch.where(fits, pages(start + add) - kept, torch.zeros_like(add))
    taken = torch.cumsum(need, 0)
    there = count + freed.sum()
    granted = fits & ((need == 0) | (taken <= there))
    # the stack of free pages, freed ones on it with the first of them on top
    b = torch.arange(len(add), device="cuda")
    i = torch.arange(table.shape[1], device="cuda")
    back = (i >= kept[:, None]) & (i < pages(lens)[:, None])
    order = torch.cumsum(freed, 0) - freed
    stack = torch.cat((s["free"], s["free"].new_zeros(1)))
    spot = torch.where(back, there - 1 - (order[:, None] + i - kept[:, None]), torch.full_like(back, len(s["free"]), dtype=torch.long))
    stack.scatter_(0, spot.flatten(), table.flatten())
    # pages from its top
    got = granted[:, None] & (i >= kept[:, None]) & (i < (kept + need)[:, None])
    spot = (there - 1 - (taken - need)[:, None] - (i - kept[:, None])).clamp(min=0, max=len(s["free"]) - 1)
    table.copy_(torch.where(got, stack[spot], table))
    left = there - torch.where(granted, need, torch.zeros_like(need)).sum()
    # entries of the list behind its end hold nothing
    end = torch.arange(len(s["free"]), device="cuda") < left
    s["free"].copy_(torch.where(end, stack[:-1], s["free"]))
    s["count"].copy_(left)
    s["lens"].copy_(torch.where(granted, start + add, start))
    cu = torch.cat((ends.new_zeros(1), ends.clamp(max=total)))
    t = torch.arange(total, device="cuda")
    row = torch.bucketize(t, cu[1:].contiguous(), right=True)
    live, row = row < len(b), row.clamp(max=len(b) - 1)
    position = start[row] + t - cu[row]
    slot = table.long()[row, (position // page).clamp(max=table.shape[1] - 1)] * page + position % page
    return {"cu": cu.int(), "positions": torch.where(live, position, torch.zeros_like(position)).int(),
            "slots": torch.where(live & granted[row], slot, torch.full_like(slot, -1)), "granted": granted.int(),
            "lens": s["lens"], "table": s["table"], "count": s["count"],
            "free": torch.where(end, s["free"], torch.full_like(s["free"], -1))}


def _plain_keep(s):
    i = torch.arange(s["path"], device="cuda")[None]
    to = s["starts"].long()[:, None] + i
    source = s["starts"].long()[:, None] + torch.where(i < s["counts"].long()[:, None], s["accepted"].long(), i)
    a, b = (s["table"].long().gather(-1, t // s["page"]) for t in (source, to))
    slot_a, slot_b = source % s["page"], to % s["page"]
    values = [s[name][a, :, slot_a] for name in ("k_codes", "v_codes", "scales")]
    s["k_codes"][b, :, slot_b], s["v_codes"][b, :, slot_b], s["scales"][b, :, slot_b] = values
    return {"k": s["k_codes"], "v": s["v_codes"], "scales": s["scales"]}


def _plain_prompt(s):
    """Queries in blocks, each over the sinks and the keys that its window reaches."""
    hk, dim, window, sinks = s["kv_heads"], s["head_dim"], s["window"], s["sinks"]
    group, block = s["heads"] // hk, min(256, s["max_q"])
    cu_q, cu_k = s["cu_q"].long(), s["cu_k"].long()
    nq, nk = cu_q[1:] - cu_q[:-1], cu_k[1:] - cu_k[:-1]
    blocks = (s["max_q"] + block - 1) // block
    i = torch.arange(blocks * block, device="cuda").view(blocks, block)
    p = i[None] + (nk - nq)[:, None, None]                                        # B, blocks, block: positions
    reach = min(window + block - 1, s["max_k"])
    last = torch.minimum(p[..., -1:], nk[:, None, None] - 1)                      # of a block's queries
    j = torch.arange(min(sinks, s["max_k"]), device="cuda").expand(*p.shape[:2], -1)
    j = torch.cat((j, last - reach + 1 + torch.arange(reach, device="cuda")), -1)  # B, blocks, keys
    twice = torch.arange(j.shape[-1], device="cuda") >= min(sinks, s["max_k"])
    real = (j >= 0) & (j < nk[:, None, None]) & ~(twice & (j < sinks))
    seen = real[:, :, None] & (j[:, :, None] <= p[..., None]) & ((p[..., None] - j[:, :, None] < window) | (j[:, :, None] < sinks))
    at_q = (cu_q[:-1, None, None] + i).clamp(max=s["q"].shape[0] - 1)
    at_k = (cu_k[:-1, None, None] + j).clamp(min=0, max=s["k"].shape[0] - 1)
    q = s["q"][at_q].float().unflatten(3, (hk, group)).permute(0, 1, 3, 4, 2, 5)    # B, blocks, hk, group, block, dim
    k = s["k"][at_k].float().permute(0, 1, 3, 4, 2)[:, :, :, None]                  # B, blocks, hk, 1, dim, keys
    v = s["v"][at_k].float().permute(0, 1, 3, 2, 4)[:, :, :, None]
    out = _softmax_product(torch.matmul(q, k) * (1 / math.sqrt(dim)), seen[:, :, None, None], v)
    out = out.permute(0, 1, 4, 2, 3, 5).flatten(1, 2).flatten(2, 3)                 # B, queries, heads, dim
    return {"out": out[i.flatten()[None] < nq[:, None]].half()}


def _plain_decode(s):
    hk, dim, batch, sinks = s["kv_heads"], s["head_dim"], s["batch"], s["sinks"]
    window = min(s["window"], s["most"]) if s["window"] else s["most"]
    if s["most"] == 0:
        return {"out": torch.zeros_like(s["q"])}
    lens = s["lens"].long()[:, None]
    sinks = min(sinks, s["most"])
    j = torch.cat((torch.arange(sinks, device="cuda").expand(batch, -1), lens - window + torch.arange(window, device="cuda")), -1)
    twice = torch.arange(sinks + window, device="cuda") >= sinks
    seen = (j >= 0) & (j < lens) & ~(twice & (j < sinks))
    k, v = (_expanded(s, s["table"], j.clamp(min=0, max=s["most"] - 1), w).permute(0, 2, 1, 3) for w in (0, 1))
    q = s["q"].float().view(batch, hk, -1, dim) * (1 / math.sqrt(dim))
    return {"out": _softmax_product(torch.matmul(q, k.transpose(2, 3)), seen[:, None, None], v).flatten(1, 2).half()}


def _plain_tree(s):
    hk, dim, batch, n = s["kv_heads"], s["head_dim"], s["batch"], s["max_q"]
    cu = s["cu_q"].long()
    nq = cu[1:] - cu[:-1]
    i = torch.arange(n, device="cuda")
    at = (cu[:-1, None] + i).clamp(max=len(s["parents"]) - 1)
    real = i < nq[:, None]
    parent = torch.where(real, s["parents"].long()[at], torch.full_like(at, -1))
    step = (parent[:, :, None] == i).float() + torch.eye(n, device="cuda")
    line = torch.linalg.matrix_power(step, 128) > 0                                 # a node's ancestors and itself
    depth = line.sum(-1) - 1
    context = (s["lens"].long() - nq)[:, None]
    j = torch.arange(s["most"], device="cuda").expand(batch, -1)
    node = (j - context).clamp(min=0, max=n - 1)                                    # of a key behind the context
    mine = j >= context
    where = torch.where(mine, context + depth.gather(-1, node), j)                  # positions of the keys
    seen = torch.where(mine[:, None], line.gather(-1, node[:, None].expand(-1, n, -1)), torch.ones_like(mine)[:, None])
    seen = seen & (j < s["lens"].long()[:, None])[:, None]
    if s["window"]:
        seen = seen & (((context + depth)[:, :, None] - where[:, None] < s["window"]) | (where < s["sinks"])[:, None])
    q = s["q"][at].float().unflatten(2, (hk, -1)).permute(0, 2, 3, 1, 4) * (1 / math.sqrt(dim))    # B, hk, group, n, dim
    group = q.shape[2]
    k, v = (_expanded(s, s["table"], j, w).permute(0, 2, 1, 3) for w in (0, 1))     # B, hk, keys, dim
    scores = torch.matmul(q.flatten(2, 3), k.transpose(2, 3))
    out = _softmax_product(scores, seen[:, None].repeat(1, 1, group, 1), v)
    return {"out": out.unflatten(2, (group, n)).permute(0, 3, 1, 2, 4).flatten(2, 3)[real].half()}


# -------------------------------------------------------- the framework's own
def _own_plan(s, spinq):
    plan = spinq.kv4_plan(s["lens"], s["add"], s["table"], s["free"], s["count"], s["page"], s["total"], drop=s["dropped"])
    return {"cu": plan.cu_tokens, "positions": plan.positions, "slots": plan.slots, "granted": plan.granted,
            "lens": s["lens"], "table": s["table"], "count": s["count"],
            "free": torch.where(torch.arange(len(s["free"]), device="cuda") < s["count"], s["free"], -1)}


def _own_keep(s, spinq):
    spinq.kv4_keep(spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"]), s["table"], s["starts"], s["accepted"], s["counts"])
    return {"k": s["k_codes"], "v": s["v_codes"], "scales": s["scales"]}


def _own_prompt(s, spinq):
    return {"out": spinq.window_prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"],
                                                 s["window"], s["sinks"])}


def _own_decode(s, spinq):
    cache = spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"])
    return {"out": spinq.window_attention_kv4(s["q"], cache, s["table"], s["lens"], s["window"], s["sinks"])}


def _own_tree(s, spinq):
    cache = spinq.KV4Pages(s["k_codes"], s["v_codes"], s["scales"])
    return {"out": spinq.tree_attention_kv4(s["q"], cache, s["table"], s["lens"], s["cu_q"], s["max_q"], s["parents"],
                                            window=s["window"], sinks=s["sinks"])}


def run(state):
    if own:
        from paper_2405_16406_gb300 import spinq
        return {"plan": _own_plan, "keep": _own_keep, "prompt": _own_prompt, "decode": _own_decode,
                "tree": _own_tree}[state["op"]](state, spinq)
    return {"plan": _plain_plan, "keep": _plain_keep, "prompt": _plain_prompt, "decode": _plain_decode,
            "tree": _plain_tree}[state["op"]](state)


# ------------------------------------------------------------ the unavoidable
def _sees(position, window, sinks):
    """How many of the tokens 0 .. position a query at `position` sees."""
    if not window:
        return position + 1
    low = max(0, position - window + 1)
    return position + 1 - low + min(sinks, low)


def work(case):
    if case["op"] == "plan":
        # lengths, drops and additions in, lengths, offsets and answers out; a position and a slot a token; a page
        # dropped is read and goes on the list, a page taken is read there and goes into the table
        n, page = sum(_lengths(case)), case["page"]
        moved = sum((case["context"] + m + page - 1) // page - (case["context"] + page - 1) // page for m in _lengths(case))
        return {"bytes": case["batch"] * 24 + (n + case["padding"]) * 12 + moved * 16, "flops": 0}
    dim, hk = case["head_dim"], case["kv_heads"]
    row4 = hk * (dim + 16)        # a token's codes and scales of K and V
    if case["op"] == "keep":
        paths = _paths(case)
        moved = sum(sum(p != i for i, p in enumerate(path)) for path in paths)
        return {"bytes": 2 * moved * row4 + sum(len(p) for p in paths) * 8 + case["batch"] * 8, "flops": 0}
    hq, window, sinks = case["heads"], case["window"], case["sinks"]
    lens = _lengths(case)
    if case["op"] == "prompt":
        pairs = sum(_sees(case["context"] + i, window, sinks) for n in lens for i in range(n))
        keys = sum(_sees(case["context"], window, sinks) + n - 1 for n in lens)
        return {"bytes": sum(lens) * hq * dim * 4 + keys * hk * dim * 4, "flops": 4 * pairs * hq * dim}
    if case["op"] == "decode":
        keys = sum(_sees(n - 1, window, sinks) for n in lens)
        return {"bytes": keys * (row4 + 4 / case["page"]) + case["batch"] * hq * dim * 4, "flops": 4 * keys * hq * dim}
    keys = pairs = nodes = 0
    for n, tree in zip(lens, _trees(case)):
        depth = []
        for p in tree:
            depth.append(0 if p < 0 else depth[p] + 1)
        nodes += len(tree)
        keys += _sees(n, window, sinks) - 1 + len(tree)
        pairs += sum(_sees(n + d, window, sinks) for d in depth)
    return {"bytes": keys * (row4 + 4 / case["page"]) + nodes * (hq * dim * 4 + 4), "flops": 4 * pairs * hq * dim}


# ------------------------------------------------------------------ 64 bits
def _exact_tokens(s, b, tokens):
    """K and V [n, Hkv, D] in 64 bits of the given tokens (a tensor) of sequence b."""
    at = s["table"][b].long()[tokens // s["page"]] * s["page"] + tokens % s["page"]
    out = []
    for which, name in ((0, "k_codes"), (1, "v_codes")):
        c = s[name].transpose(1, 2).flatten(0, 1)[at].int()
        f = s["scales"].transpose(1, 2).flatten(0, 1)[at].double()
        u = torch.empty(c.shape[:2] + (s["head_dim"],), dtype=torch.float64, device="cuda")
        u[..., 0::2], u[..., 1::2] = (c % 16).double(), (c // 16).double()
        out.append(u * f[..., 2 * which:2 * which + 1] + f[..., 2 * which + 1:2 * which + 2])
    return out


def _exact_attention(q, k, v, seen=None):
    """q [n, Hq, D], k and v [m, Hkv, D] in 64 bits; seen [n, m] or None.  Every query sees a key, or there is none."""
    out = torch.zeros_like(q)
    if k.shape[0] == 0:
        return out
    group = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        a = q[:, h] @ k[:, h // group].T / math.sqrt(q.shape[-1])
        if seen is not None:
            a = a.masked_fill(~seen, -math.inf)
        out[:, h] = torch.softmax(a, -1) @ v[:, h // group]
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return None   # whole numbers
    s = prepare(case, seed)
    if case["op"] == "keep":
        scales, table = s["scales"].double().cpu(), s["table"].cpu()
        for b, path in enumerate(_paths(case)):
            at = [(int(table[b, (case["context"] + p) // s["page"]]), (case["context"] + p) % s["page"])
                  for p in range(case["nodes"])]
            rows = [scales[at[p][0], :, at[p][1]].clone() for p in path]
            for i, row in enumerate(rows):
                scales[at[i][0], :, at[i][1]] = row
        return {"k": None, "v": None, "scales": scales}
    window, sinks, lens = case["window"], case["sinks"], _lengths(case)
    dev = torch.device("cuda")
    if case["op"] == "prompt":
        out, at, ak = [], 0, 0
        for n in lens:
            m, c = n + case["context"], case["context"]
            for a in range(0, n, 1024):
                e = min(n, a + 1024)
                first = max(0, c + a - window + 1)
                j = torch.cat((torch.arange(min(sinks, first), device=dev), torch.arange(first, c + e, device=dev)))
                p = torch.arange(c + a, c + e, device=dev)[:, None]
                seen = (j <= p) & ((j > p - window) | (j < sinks))
                out.append(_exact_attention(s["q"][at + a:at + e].double(), s["k"][ak + j].double(), s["v"][ak + j].double(), seen))
            at, ak = at + n, ak + m
        return {"out": torch.cat(out)}
    if case["op"] == "decode":
        out = []
        for b, n in enumerate(lens):
            first = max(0, n - window) if window else 0
            j = torch.cat((torch.arange(min(sinks, first), device=dev), torch.arange(first, n, device=dev)))
            out.append(_exact_attention(s["q"][b:b + 1].double(), *_exact_tokens(s, b, j)))
        return {"out": torch.cat(out)}
    out, at = [], 0
    for b, (n, tree) in enumerate(zip(lens, _trees(case))):
        lines = []
        for i, p in enumerate(tree):
            lines.append((lines[p] if p >= 0 else []) + [i])
        first = max(0, n - window) if window else 0
        j = torch.cat((torch.arange(min(sinks, first), device=dev), torch.arange(first, n + len(tree), device=dev)))
        place = torch.cat((torch.arange(n), n - 1 + torch.tensor([len(x) for x in lines]))).to(dev)[j]
        seen = torch.zeros((len(tree), n + len(tree)), dtype=torch.bool)
        seen[:, :n] = True
        for i, line in enumerate(lines):
            seen[i, [n + x for x in line]] = True
        seen = seen.to(dev)[:, j]
        if window:
            here = (n - 1 + torch.tensor([len(x) for x in lines], device=dev))[:, None]
            seen &= (place > here - window) | (place < sinks)
        out.append(_exact_attention(s["q"][at:at + len(tree)].double(), *_exact_tokens(s, b, j), seen))
        at += len(tree)
    return {"out": torch.cat(out)}
