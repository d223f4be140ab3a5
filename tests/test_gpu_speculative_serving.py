"""The operators of drafted trees and windows together, as a server uses them.

Bar of the outputs: attention on the codes against fp64 attention over the
read-back fp16 K and V.  K and V are rounded to fp16 by the read-back (2^-11 each,
the scores by 2^-11 of |q| |k| scale), the kernel rounds the output (2^-11): under
2^-8 in norm.  Bookkeeping and moved tokens: equal."""
import os
import random
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("kw", [dict(requests=5, steps=4), dict(requests=20, steps=3, heads=8, kv_heads=8, dim=64, page=16),
                                dict(requests=7, steps=5, window=100, sinks=3), dict(requests=3, steps=2, most_nodes=60, page=256)])
def test_example_verifies_what_the_read_back_cache_says(kw):
    import speculative_serving as ex
    from paper_2405_16406_gb300 import spinq
    out, q, trees, layer, plan = ex.serve(**kw)
    assert plan.granted.all()
    ref = ex.attention_over_read_back(q, trees, layer, plan, kw.get("window", 0), kw.get("sinks", 4))
    assert float((out.double() - ref).norm() / ref.norm()) < 2.0 ** -8
    held = sum(-(-n // layer.page) for n in layer.lens.tolist())
    assert held + layer.count.item() == layer.free.numel(), "every page is a sequence's or free"
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK


def test_a_kept_path_is_what_appending_it_alone_gives():
    """Draft a tree, keep a path, drop the rest: the cache reads as if the path's tokens had been appended one after
    another, and the next token attends to the same."""
    import speculative_serving as ex
    from paper_2405_16406_gb300 import spinq
    rng = random.Random(3)
    g = torch.Generator(device="cuda").manual_seed(5)
    width = (8 + 2 * 2) * 128
    prompts, nodes = [70, 5, 129], 17
    fused = torch.randn((sum(prompts), width), generator=g, device="cuda").half()
    drafts = torch.randn((3 * nodes, width), generator=g, device="cuda").half()
    trees = [ex.draft(rng, nodes) for _ in range(3)]
    paths = [ex.choose(rng, p) for p, _ in trees]
    layers = [ex.Layer(3, 400, 8, 2, 128, 16, seed=s) for s in (0, 1)]
    for layer in layers:
        layer.append(fused, layer.plan(ex.ints(prompts), sum(prompts)))
    a, b = layers
    plan = a.plan(ex.ints([nodes] * 3), 3 * nodes, depths=ex.ints([d for _, t in trees for d in t]))
    a.append(drafts, plan)
    deepest = max(map(len, paths))
    spinq.kv4_keep(a.cache, a.table, a.lens - nodes, ex.ints([p + [0] * (deepest - len(p)) for p in paths]),
                   ex.ints([len(p) for p in paths]))
    a.plan(None, 0, drop=ex.ints([nodes - len(p) for p in paths]))
    rows = torch.tensor([nodes * i + x for i, p in enumerate(paths) for x in p], device="cuda")
    b.append(drafts[rows], b.plan(ex.ints([len(p) for p in paths]), len(rows)))
    assert a.lens.tolist() == b.lens.tolist() == [n + len(p) for n, p in zip(prompts, paths)]
    cu, total = ex.offsets(a.lens.tolist()), int(a.lens.sum())
    for x, y in zip(spinq.kv4_read(a.cache, a.table, cu, total), spinq.kv4_read(b.cache, b.table, cu, total)):
        assert torch.equal(x, y)
    q = torch.randn((3, 8, 128), generator=g, device="cuda").half()
    for w in (0, 20):
        x, y = (spinq.window_attention_kv4(q, layer.cache, layer.table, layer.lens, w, 2) for layer in layers)
        assert torch.equal(x, y)


def test_a_step_replays_from_one_graph():
    """Plan, append, attention and keep of a step captured once, replayed with other lengths: the same as without a
    graph."""
    import speculative_serving as ex
    from paper_2405_16406_gb300 import spinq
    nodes, B = 8, 4
    layers = [ex.Layer(B, 500, 8, 2, 64, 16, seed=0) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    fused = torch.randn((100, 12 * 64), generator=g, device="cuda").half()
    for layer in layers:
        layer.append(fused, layer.plan(ex.ints([40, 3, 30, 27]), 100))
    rng = random.Random(9)
    trees = [ex.draft(rng, nodes) for _ in range(B)]
    parents, depths = ex.ints([x for p, _ in trees for x in p]), ex.ints([x for _, d in trees for x in d])
    path, counts, add = ex.ints([[0, 2, 5], [0, 1, 0], [0, 0, 0], [0, 3, 7]]), ex.ints([3, 2, 1, 3]), ex.ints([nodes] * B)
    drafts = torch.zeros((B * nodes, 12 * 64), dtype=torch.float16, device="cuda")
    drop = torch.zeros(B, dtype=torch.int32, device="cuda")

    def step(layer):
        plan = layer.plan(add, B * nodes, drop=drop, depths=depths)
        q = layer.append(drafts, plan)
        out = spinq.tree_attention_kv4(q, layer.cache, layer.table, layer.lens, plan.cu_tokens, nodes, parents)
        spinq.kv4_keep(layer.cache, layer.table, layer.lens - nodes, path, counts)
        return out

    state = [x.clone() for x in (layers[0].lens, layers[0].table, layers[0].free, layers[0].count)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(layers[0])
    for x, y in zip((layers[0].lens, layers[0].table, layers[0].free, layers[0].count), state):
        assert torch.equal(x, y), "capturing runs nothing"
    for k in range(4):
        drafts.copy_(torch.randn(drafts.shape, generator=g, device="cuda").half())
        drop.copy_((nodes - counts) if k else torch.zeros_like(drop))
        graph.replay()
        want = step(layers[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert layers[0].lens.tolist() == layers[1].lens.tolist() and torch.equal(layers[0].table, layers[1].table)
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
