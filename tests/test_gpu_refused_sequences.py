"""A server's steps in which pages run out: what a refused sequence's rows give means
nothing, but the others' outputs are right, every page and the refused sequence's own
tokens are as they were, and it is served as soon as there are pages."""
import copy
import os
import random
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("nodes", [2, 6, 20])   # 8, 24 and 80 rows of a kv head
def test_refused_beside_served(nodes):
    import speculative_serving as ex
    from paper_2405_16406_gb300 import spinq
    rng = random.Random(nodes)
    g = torch.Generator(device="cuda").manual_seed(nodes)
    project = lambda n: torch.randn((n, (8 + 4) * 128), generator=g, device="cuda").half()   # noqa: E731
    layer = ex.Layer(4, 200, 8, 2, 128, 16)
    # prompts of 3, 4, 3 and 5 full pages leave one page
    layer.count.fill_(16)
    prompts = [48, 64, 48, 80]
    layer.append(project(240), layer.plan(ex.ints(prompts), 240))
    assert layer.count.item() == 1 and layer.lens.tolist() == prompts
    trees = [ex.draft(rng, min(nodes, 16)), ([], []), ex.draft(rng, nodes), ex.draft(rng, nodes)]
    sizes = [len(p) for p, _ in trees]
    depths, parents = ex.ints([d for _, t in trees for d in t]), ex.ints([x for p, _ in trees for x in p])
    before = [x.clone() for x in (layer.cache.k_codes, layer.cache.v_codes, layer.cache.scales)]

    def step(drop=None):
        plan = layer.plan(ex.ints(sizes), sum(sizes), drop=drop, depths=depths)
        q = layer.append(project(sum(sizes)), plan)
        out = spinq.tree_attention_kv4(q, layer.cache, layer.table, layer.lens, plan.cu_tokens, max(sizes), parents)
        torch.cuda.synchronize()
        return plan, q, out

    def near(out, q, which):   # the sequences of these rows
        part = copy.copy(layer)
        part.lens, part.table = layer.lens[which], layer.table[which]
        # (read-back K and V rounded to fp16, and the output: under 2^-8 in norm)
        ref = ex.attention_over_read_back(q, [trees[b] for b in which], part, None, 0, 0)
        return float((out.double() - ref).norm() / ref.norm()) < 2.0 ** -8

    plan, q, out = step()
    assert plan.granted.tolist() == [1, 1, 0, 0] and layer.lens.tolist() == [48 + sizes[0], 64, 48, 80]
    assert near(out[:sizes[0]], q, [0])
    held = [p for b, n in enumerate(layer.lens.tolist()) for p in layer.table[b, :-(-n // 16)].tolist()]
    assert len(set(held)) == len(held) == 16 and layer.count.item() == 0
    old = [p for p in held if p != int(layer.table[0, 3])]
    for x, y in zip((layer.cache.k_codes, layer.cache.v_codes, layer.cache.scales), before):
        assert torch.equal(x[old].view(torch.uint8), y[old].view(torch.uint8)), "the prompts' tokens"
    # the roots are kept, of a refused sequence nothing is kept or dropped
    kept = ex.ints([1, 0, 1, 1])
    spinq.kv4_keep(layer.cache, layer.table, layer.lens - ex.ints(sizes), ex.ints([[0]] * 4), kept * plan.granted)
    drop = (ex.ints(sizes) - kept) * plan.granted
    # pages come back: all are served
    layer.free[:8] = ex.ints([p for p in range(layer.free.numel()) if p not in held][:8])
    layer.count.fill_(8)
    plan, q, out = step(drop)
    assert plan.granted.all() and layer.lens.tolist() == [49 + sizes[0], 64, 48 + sizes[2], 80 + sizes[3]]
    assert near(out, q, [0, 2, 3])   # (sequence 1 has no rows)
    assert spinq.spinq_device_status()[0] == spinq.SPINQ_OK
