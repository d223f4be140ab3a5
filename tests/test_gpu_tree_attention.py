"""spinq_tree_attention_kv4 and spinq_window_attention_kv4 on the GPU against
attention in 64 bits over the same codes and scales.

Bar, per value: scores (base 2) are fp32 sums of terms of at most 64 or so: off by
less than 2^-15 (64 times a few 2^-23), so a weight and the sum that divides it
by less than 2^-15 each; the weights as two fp16 parts by 2^-21; the output once, by
half a step: |err| <= 2^-13 sum_j p_j |v_j| + 2^-11 |o| + 2^-24."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def _bar(o, size):
    return 2.0 ** -13 * size + 2.0 ** -11 * np.abs(o) + 2.0 ** -24


def forest(rng, n, roots=0.1):
    """Parents of n nodes, some of them roots."""
    return [-1 if i == 0 or rng.random() < roots else int(rng.integers(max(0, i - 7), i)) for i in range(n)]


def lines_of(parents):
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def visible(parents, n, window, sinks):
    """[nq, n]: what each query sees of the sequence's n tokens, the last len(parents) of them its own."""
    nq = len(parents)
    ctx = n - nq
    lines = lines_of(parents)
    place = {j: j for j in range(max(ctx, 0))}
    seen = np.zeros((nq, max(n, 0)), bool)
    for i, line in enumerate(lines):
        here = ctx + len(line) - 1
        for j in range(max(ctx, 0)):
            seen[i, j] = not window or here - j < window or j < sinks
        for x in line:
            there = ctx + len(lines[x]) - 1
            if ctx + x >= 0 and (not window or here - there < window or there < sinks):
                seen[i, ctx + x] = True
    return seen


def build(S, lens, Hkv, D, P, seed, window=0, sinks=0, nodes=None, extra_width=0):
    """A cache whose slots that nothing sees are NaN, with pages given back as -1: page 0 holds NaN scales."""
    rng = np.random.default_rng(seed)
    table, pages = ku.page_tables(rng, lens, P)
    table = np.where(table >= 0, table + 1, table)
    cache = ku.random_cache(S, rng, pages + 1, P, Hkv, D)
    sc = cache.scales
    written = torch.zeros((pages + 1, P), dtype=torch.bool)
    for b, n in enumerate(lens):
        for i in range(-(-n // P)):
            written[table[b, i], :min(P, n - i * P)] = True
    sc.masked_fill_(~written.cuda()[:, None, :, None], float("nan"))
    full = table.copy()
    if window:
        for b, n in enumerate(lens):
            first = max(0, n - (nodes[b] if nodes else 1) - window + 1)
            for i in range(first // P):
                if i * P >= sinks:
                    sc[int(table[b, i])] = float("nan")
                    table[b, i] = [-1, 0, 2 ** 31 - 1][i % 3] if pages else -1
                    if table[b, i] == 2 ** 31 - 1:
                        table[b, i] = -5
    if extra_width:
        table = np.concatenate([table, np.full((len(lens), extra_width), -1, np.int32)], 1)
    return rng, cache, table.astype(np.int32), full


def reference(cache, table, q, n, seen, P, scale):
    """o, sum p |v| of q [nq, Hq, D] over the n tokens of a page list."""
    (ku_, ka, kb), (vu, va, vb) = ku.slot_values(cache, ku.token_slots(table, P, 0, n))
    k, v = ku_ * ka[..., None] + kb[..., None], vu * va[..., None] + vb[..., None]
    any_row = seen.any(0)
    return ku.attention(q.astype(np.float64), k[any_row], v[any_row], scale, seen[:, any_row])


def run_tree(S, ctx, trees, Hq, Hkv, D, P, window=0, sinks=0, seed=0, scale=None, slack=0, extra_width=0, spread=2.0, pad=3, **kw):
    """ctx: context lengths (below 0: the cache lacks that many of the first queries' tokens)."""
    nodes = [len(t) for t in trees]
    lens = [max(c + n, 0) for c, n in zip(ctx, nodes)]
    rng, cache, table, full = build(S, lens, Hkv, D, P, seed, window, sinks, nodes, extra_width)
    T = sum(nodes)
    q = (rng.standard_normal((T + pad, Hq, D)) * spread).astype(np.float16)
    cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()   # noqa: E731
    out = torch.full((T + pad, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    parents = dev(np.array([p for t in trees for p in t] + [0] * pad, np.int32))
    torch.cuda.synchronize()
    S.tree_attention_kv4(dev(q), cache, dev(table), dev(np.array(lens, np.int32)), dev(cu), max(nodes + [1]) + slack, parents,
                         window, sinks, scale=scale, out=out, **kw)
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    assert np.all(got[T:] == 7.0), "rows behind the last sequence are not written"
    for b, t in enumerate(trees):
        if not t:
            continue
        seen = visible(t, ctx[b] + len(t), window, sinks)[:, :lens[b]]
        o, size = reference(cache, full[b], q[cu[b]:cu[b + 1]], lens[b], seen, P, 1 / np.sqrt(D) if scale is None else scale)
        err = np.abs(got[cu[b]:cu[b + 1]] - o)
        assert np.all(err <= _bar(o, size)), (b, float((err - _bar(o, size)).max()))
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 2), (40, 5), (130, 70), (500, 0)])
@pytest.mark.parametrize("ctx,nodes,Hq,Hkv,P", [
    ([0], [1], 8, 8, 16),
    ([5, 64, 63, 65], [1, 1, 2, 1], 8, 2, 16),
    ([100, 0, 17, 300], [4, 3, 0, 8], 8, 2, 32),
    ([200, 31], [16, 9], 8, 1, 64),
    ([700, 1, 128], [33, 20, 64], 8, 2, 128),
    ([257, 640], [128, 100], 4, 2, 256),
])
def test_matches_64_bits(S, D, window, sinks, ctx, nodes, Hq, Hkv, P):
    rng = np.random.default_rng(sum(ctx) + D)
    run_tree(S, ctx, [forest(rng, n) for n in nodes], Hq, Hkv, D, P, window, sinks, seed=sum(nodes))


@pytest.mark.parametrize("Hq,Hkv", [(3, 1), (7, 1), (10, 2), (17, 1), (71, 1), (128, 1), (24, 8)])
def test_head_groups_of_any_size(S, Hq, Hkv):
    rng = np.random.default_rng(Hq)
    run_tree(S, [90, 333], [forest(rng, n) for n in (7, 20)], Hq, Hkv, 64, 16, seed=Hq)
    run_tree(S, [90, 333], [forest(rng, n) for n in (1, 2)], Hq, Hkv, 128, 16, 50, 3, seed=Hq)


def test_chains_and_trees_of_one_line(S):
    """No parents: a chain, bit by bit what its parents give."""
    rng = np.random.default_rng(0)
    lens = [150, 20, 7]
    _, cache, table, _ = build(S, lens, 2, 128, 32, 1)
    q = torch.from_numpy(rng.standard_normal((20, 8, 128)).astype(np.float16)).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    cu, parents = i32([0, 9, 13, 20]), i32(list(range(-1, 8)) + [-1, 0, 1, 2] + list(range(-1, 6)))
    for w in (0, 4):
        a = S.tree_attention_kv4(q, cache, torch.from_numpy(table).cuda(), i32(lens), cu, 9, None, w, 1)
        b = S.tree_attention_kv4(q, cache, torch.from_numpy(table).cuda(), i32(lens), cu, 9, parents, w, 1)
        torch.cuda.synchronize()
        assert torch.equal(a, b)


def test_parents_that_are_none(S):
    """Any number that is no earlier node makes a root."""
    rng = np.random.default_rng(3)
    good = [-1, 0, -1, 2, -1, 4]
    lens = [70]
    _, cache, table, _ = build(S, lens, 2, 64, 16, 2)
    q = torch.from_numpy(rng.standard_normal((6, 4, 64)).astype(np.float16)).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    call = lambda p: S.tree_attention_kv4(q, cache, torch.from_numpy(table).cuda(), i32(lens), i32([0, 6]), 6, i32(p))   # noqa: E731
    a = call(good)
    for bad in ([0, 0, 2, 2, 5, 4], [7, 0, 99, 2, 2 ** 31 - 1, 4], [-2 ** 31, 0, -9, 2, 4, 4]):
        b = call(bad)
        torch.cuda.synchronize()
        assert torch.equal(a, b)


def test_queries_whose_tokens_are_not_in_the_cache(S):
    """Lengths below the number of queries: what is missing is not seen, a query without any key gives zeros."""
    rng = np.random.default_rng(4)
    for w, s in ((0, 0), (2, 0), (3, 9)):
        out = run_tree(S, [-3, -5, 40], [[-1, 0, 0, 1, 2], forest(rng, 5), [-1]], 8, 2, 64, 16, w, s)
        assert not out[5:10].any()


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_numbers_stay_with_who_sees_them(S, D):
    """A drafted token with NaN scales, and one with infinite ones: its descendants' rows, no others."""
    rng = np.random.default_rng(5)
    tree = [-1, 0, 0, 1, 2, 4, 3, 1]
    lens = [100 + 8]
    for nq_heads in (2, 16):   # both row counts
        _, cache, table, _ = build(S, lens, 2, D, 16, 3)
        q = torch.from_numpy(rng.standard_normal((8, nq_heads, D)).astype(np.float16)).cuda()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        call = lambda: S.tree_attention_kv4(q, cache, torch.from_numpy(table).cuda(), i32(lens), i32([0, 8]), 8, i32(tree))   # noqa: E731
        clean = call()
        for bad in (float("nan"), float("inf")):
            kept = cache.scales.clone()
            t = 100 + 2
            cache.scales[int(table[0, t // 16]), :, t % 16] = bad
            dirty = call()
            torch.cuda.synchronize()
            cache.scales.copy_(kept)
            below = [i for i, line in enumerate(lines_of(tree)) if 2 in line]
            rest = [i for i in range(8) if i not in below]
            assert torch.equal(clean[rest], dirty[rest])
            assert dirty[below].isnan().all()


def test_a_query_that_is_not_a_number_gives_its_own_row_only(S):
    rng = np.random.default_rng(6)
    _, cache, table, _ = build(S, [300, 70], 2, 128, 16, 4)
    q = torch.from_numpy(rng.standard_normal((30, 8, 128)).astype(np.float16)).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    call = lambda: S.tree_attention_kv4(q, cache, torch.from_numpy(table).cuda(), i32([300, 70]), i32([0, 20, 30]), 20)   # noqa: E731
    clean = call()
    q[7, 3, 5] = float("nan")
    q[21, 6, 0] = float("inf")
    out = call()
    torch.cuda.synchronize()
    bad = torch.zeros(30, 8, dtype=torch.bool, device="cuda")
    bad[7, 3] = bad[21, 6] = True
    assert out[7, 3].isnan().all() and torch.equal(out[~bad], clean[~bad])


def test_large_scores_and_scales(S):
    rng = np.random.default_rng(7)
    run_tree(S, [600], [forest(rng, 9)], 8, 2, 128, 64, scale=0.0)
    run_tree(S, [600], [forest(rng, 40)], 8, 2, 128, 64, scale=-0.1, spread=1.0)


def test_lengths_far_under_the_planned_maximum(S):
    rng = np.random.default_rng(8)
    run_tree(S, [30, 7], [forest(rng, 2), forest(rng, 3)], 8, 2, 128, 16, slack=100, extra_width=500)


def test_many_sequences_of_all_lengths(S):
    rng = np.random.default_rng(9)
    ctx = rng.integers(0, 400, 150).tolist()
    run_tree(S, ctx, [forest(rng, int(n)) for n in rng.integers(0, 6, 150)], 4, 2, 64, 16, seed=1)
    run_tree(S, ctx[:40], [forest(rng, int(n)) for n in rng.integers(0, 50, 40)], 8, 2, 128, 32, 100, 7, seed=2)


def test_long_contexts(S):
    rng = np.random.default_rng(10)
    run_tree(S, [9001, 3], [forest(rng, 12), forest(rng, 30)], 8, 2, 128, 64)
    run_tree(S, [30000], [[-1]], 4, 1, 128, 256)
    run_tree(S, [6000, 100], [forest(rng, 60), forest(rng, 128)], 4, 1, 64, 16, 4096, 4)


def test_same_result_every_time_on_any_stream_and_in_graphs(S):
    """Two captured graphs with a workspace each, replayed with new lengths."""
    rng = np.random.default_rng(11)
    _, cache, table, _ = build(S, [900, 64, 333], 2, 128, 16, 5)
    table = torch.from_numpy(table).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    for n, G in ((3, 4), (40, 4)):
        q = torch.from_numpy(rng.standard_normal((3 * n, 2 * G, 128)).astype(np.float16)).cuda()
        cu, lens = i32([0, n, 2 * n, 3 * n]), i32([900, 64, 333])
        call = lambda **kw: S.tree_attention_kv4(q, cache, table, lens, cu, n, **kw)   # noqa: E731
        first = call()
        torch.cuda.synchronize()
        second = call(stream=torch.cuda.Stream())
        torch.cuda.synchronize()
        assert torch.equal(first, second)
        graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], [torch.zeros_like(first), torch.zeros_like(first)]
        need = S.spinq_tree_attention_workspace_bytes(3, n, table.shape[1], 16, 2 * G, 2, 128)
        spaces = [torch.zeros(need, dtype=torch.uint8, device="cuda") for _ in graphs]
        for g, o, w in zip(graphs, outs, spaces):
            with torch.cuda.graph(g):
                call(out=o, workspace=w)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, outs[0]) and torch.equal(first, outs[1])
        lens.copy_(i32([500, 40, 300]))
        again = call()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(again, outs[1]) and not torch.equal(again, first)


# ------------------------------------------------------------ one query each
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (64, 4), (100, 200), (1000, 17)])
@pytest.mark.parametrize("lens,Hq,Hkv,P", [([1], 8, 8, 16), ([0, 1, 16, 17, 64, 65], 8, 2, 16), ([900, 0, 2500, 77], 32, 8, 64),
                                           ([300, 299], 20, 2, 256), ([129, 1], 71, 1, 32)])
def test_one_query_each(S, D, window, sinks, lens, Hq, Hkv, P):
    rng, cache, table, full = build(S, lens, Hkv, D, P, len(lens) + D, window, sinks)
    q = (rng.standard_normal((len(lens), Hq, D)) * 2).astype(np.float16)
    dev = lambda x: torch.from_numpy(x).cuda()   # noqa: E731
    out = S.window_attention_kv4(dev(q), cache, dev(table), dev(np.array(lens, np.int32)), window, sinks)
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    for b, n in enumerate(lens):
        if n == 0:
            assert not got[b].any()
            continue
        seen = visible([-1], n, window, sinks)
        o, size = reference(cache, full[b], q[b:b + 1], n, seen, P, 1 / np.sqrt(D))
        assert np.all(np.abs(got[b] - o[0]) <= _bar(o[0], size[0])), b
    assert S.spinq_device_status()[0] == S.SPINQ_OK


def test_lengths_out_of_range_are_clamped(S):
    _, cache, table, _ = build(S, [128, 128], 2, 64, 16, 9)
    q = torch.from_numpy(np.random.default_rng(0).standard_normal((2, 8, 64)).astype(np.float16)).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    t = torch.from_numpy(table).cuda()
    a = S.window_attention_kv4(q, cache, t, i32([128, 0]), 50, 2)
    b = S.window_attention_kv4(q, cache, t, i32([2 ** 31 - 1, -5]), 50, 2)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_one_query_is_a_tree_of_one(S):
    _, cache, table, _ = build(S, [300, 20], 2, 128, 16, 10)
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((2, 8, 128)).astype(np.float16)).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    t = torch.from_numpy(table).cuda()
    a = S.window_attention_kv4(q, cache, t, i32(300, 20), 100, 2)
    b = S.tree_attention_kv4(q, cache, t, i32(300, 20), i32(0, 1, 2), 1, i32(-1, -1), 100, 2)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
