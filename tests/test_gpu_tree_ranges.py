"""Tree and window attention, kept paths and the page plan where numbers get large: a cache past 2^32 bytes,
value scales far apart, calls on two streams at once, sequences that the plan refused."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_pages_behind_4_gib(S):
    """The same tokens in the first pages of a small cache and in the last of one of 150000 pages (4.9 GB of key
    codes): equal outputs, equal moved tokens."""
    rng = np.random.default_rng(0)
    small = ku.random_cache(S, rng, 12, 64, 8, 128)
    big = S.kv4_pages(150000, 64, 8, 128)
    assert big.k_codes.numel() > 1 << 32
    last = 150000 - 12
    for x, y in ((big.k_codes, small.k_codes), (big.v_codes, small.v_codes), (big.scales, small.scales)):
        x[last:] = y
    order = rng.permutation(12).astype(np.int32).reshape(2, 6)
    tables = [torch.from_numpy(order).cuda(), torch.from_numpy(order + last).cuda()]
    for nodes in (1, 5, 20, 60):
        q = torch.from_numpy(rng.standard_normal((2 * nodes, 32, 128)).astype(np.float16)).cuda()
        lens = i32([384, 300])
        a, b = (S.tree_attention_kv4(q, c, t, lens, i32([0, nodes, 2 * nodes]), nodes) for c, t in zip((small, big), tables))
        torch.cuda.synchronize()
        assert torch.equal(a, b)
    for c, t in zip((small, big), tables):
        S.kv4_keep(c, t, i32([370, 290]), i32([[1, 5, 9], [0, 3, 8]]), i32([3, 3]))
    torch.cuda.synchronize()
    assert torch.equal(big.k_codes[last:], small.k_codes) and torch.equal(big.v_codes[last:], small.v_codes)
    assert torch.equal(big.scales[last:], small.scales)
    assert S.spinq_device_status()[0] == S.SPINQ_OK


@pytest.mark.parametrize("nodes", [1, 4, 12, 40])
@pytest.mark.parametrize("low,high", [(-20, 0), (0, 12), (-30, 10)])
def test_value_scales_far_apart(S, nodes, low, high):
    """Scales of the values 2^low .. 2^high.  Bar as test_gpu_tree_attention.py's: the weights are relative to the
    largest p alpha', so one below 2^-24 of it may lose its second part: 2^-25 of the largest p alpha' times 15 steps per
    token, 2^-14 of the row's size for 128 tokens, half of what the bar holds for the weights."""
    rng = np.random.default_rng(nodes)
    n, P, D = 128, 16, 128
    cache = ku.random_cache(S, rng, 9, P, 2, D)
    alpha = torch.from_numpy(2.0 ** rng.uniform(low, high, (9, 2, P))).float().cuda()
    cache.scales[..., 2] = alpha
    cache.scales[..., 3] = -7.5 * alpha
    table = rng.permutation(9)[:8].astype(np.int32)
    q = (rng.standard_normal((nodes, 8, D)) * 0.5).astype(np.float16)
    out = S.tree_attention_kv4(torch.from_numpy(q).cuda(), cache, torch.from_numpy(table[None]).cuda(), i32([n]),
                               i32([0, nodes]), nodes)
    torch.cuda.synchronize()
    (k, ka, kb), (v, va, vb) = ku.slot_values(cache, ku.token_slots(table, P, 0, n))
    seen = np.arange(n)[None] <= np.arange(nodes)[:, None] + n - nodes
    o, size = ku.attention(q.astype(np.float64), k * ka[..., None] + kb[..., None], v * va[..., None] + vb[..., None],
                           1 / np.sqrt(D), seen)
    # sum_j p_j |alpha_j| 15, what the steps' rounding is relative to
    _, steps = ku.attention(q.astype(np.float64), k * ka[..., None] + kb[..., None],
                            np.broadcast_to(15 * va[..., None], v.shape), 1 / np.sqrt(D), seen)
    err = np.abs(out.cpu().numpy().astype(np.float64) - o)
    bar = 2.0 ** -13 * np.maximum(size, steps) + 2.0 ** -11 * np.abs(o) + 2.0 ** -24
    assert np.all(err <= bar), float((err - bar).max())


def test_two_streams_at_once(S):
    rng = np.random.default_rng(1)
    cache = ku.random_cache(S, rng, 300, 64, 8, 128)
    table = torch.from_numpy(rng.permutation(300).astype(np.int32).reshape(3, 100)).cuda()
    lens = i32([6000, 40, 3333])
    calls = []
    for nodes in (1, 40, 8, 2):
        q = torch.from_numpy(rng.standard_normal((3 * nodes, 32, 128)).astype(np.float16)).cuda()
        cu = i32([0, nodes, 2 * nodes, 3 * nodes])
        calls.append(lambda st=None, q=q, cu=cu, n=nodes: S.tree_attention_kv4(q, cache, table, lens, cu, n, stream=st))
    want = [f() for f in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [f(st) for f, st in zip(calls, streams)]
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert torch.equal(x, y)


def test_tokens_of_a_refused_sequence_are_not_written(S):
    """Pages for one of two sequences: the other's tokens have slots -1 and the cache is as it was there."""
    cache = S.kv4_pages(3, 16, 1, 64)
    for x in (cache.k_codes, cache.v_codes, cache.scales):
        x.zero_()
    lens, table = i32([0, 0]), torch.full((2, 2), -1, dtype=torch.int32, device="cuda")
    free, count = i32([2, 0, 1]), i32([2])
    plan = S.kv4_plan(lens, i32([20, 17]), table, free, count, 16, 37)
    k, v = (torch.randn((37, 1, 64), device="cuda").half() for _ in range(2))
    S.kv4_append(None, k, v, cache, plan.slots)
    torch.cuda.synchronize()
    assert plan.granted.tolist() == [1, 0] and lens.tolist() == [20, 0] and count.item() == 0
    assert table.tolist() == [[0, 2], [-1, -1]] and (plan.slots[20:] == -1).all()
    assert not cache.scales[1].any() and cache.scales[0].any() and cache.scales[2, :, :4].any() and not cache.scales[2, :, 4:].any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [(2500,), (5130,), (20479,), (12000, 77)])
def test_few_jobs_of_long_contexts(S, D, lens):
    """One kv head: the runs end where a job has as many parts as are joined.  Each row against its own
    attention over the keys that the pages hold."""
    rng = np.random.default_rng(sum(lens) + D)
    P = 64
    table, pages = ku.page_tables(rng, list(lens), P)
    cache = ku.random_cache(S, rng, pages, P, 1, D)
    for G in (1, 3, 8, 16):
        q = (rng.standard_normal((len(lens), G, D)) * 2).astype(np.float16)
        got = S.window_attention_kv4(torch.from_numpy(q).cuda(), cache, torch.from_numpy(table.astype(np.int32)).cuda(),
                                     i32(list(lens)), 0, 0).cpu().numpy().astype(np.float64)
        for b, n in enumerate(lens):
            (ku_, ka, kb), (vu, va, vb) = ku.slot_values(cache, ku.token_slots(table[b], P, 0, n))
            k, v = ku_ * ka[..., None] + kb[..., None], vu * va[..., None] + vb[..., None]
            o, size = ku.attention(q[b:b + 1].astype(np.float64), k, v, 1 / np.sqrt(D), np.ones((1, n), bool))
            # (the output's rounding to fp16 is 2^-11 |o|; weights and sums are within 2^-13 of sum p |v|)
            assert np.all(np.abs(got[b] - o[0]) <= 2.0 ** -13 * size[0] + 2.0 ** -11 * np.abs(o[0]) + 2.0 ** -24), (G, b)
    assert S.spinq_device_status()[0] == S.SPINQ_OK


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (70, 3), (300, 130), (1000, 4), (5000, 700)])
def test_many_jobs_of_few_rows(S, D, P, window, sinks):
    """Batches whose warps take 64 tokens a step: lengths around its, the units' and the pages' ends, windows that
    leave steps and sinks in the middle of one; pages that no row sees hold numbers that are not."""
    import test_gpu_tree_attention as trees
    rng = np.random.default_rng(P + window + D)
    ctx = [0, 1, 14, 15, 16, 30, 31, 47, 62, 63, 64, 127, 128, 191, 254, 255, 256, 257, 511, 700, 1023, 1500, 2047, 3001]
    for nodes, Hq, Hkv in (([1] * 24, 4, 1), ([int(n) for n in rng.integers(0, 5, 24)], 2, 1),
                           ([int(n) for n in rng.integers(1, 3, 24)], 6, 2)):
        trees.run_tree(S, ctx, [trees.forest(rng, n) for n in nodes], Hq, Hkv, D, P, window, sinks, seed=P + sum(nodes))


def test_few_jobs_and_many(S):
    """A sequence alone and among copies of itself: other steps and parts, each within the bound of the
    attention in 64 bits."""
    import test_gpu_tree_attention as trees
    rng = np.random.default_rng(5)
    cache = ku.random_cache(S, rng, 80, 64, 1, 128)
    row = rng.permutation(80).astype(np.int32)
    q = rng.standard_normal((1, 4, 128)).astype(np.float16)
    for window, sinks in ((0, 0), (900, 70)):
        o, size = trees.reference(cache, row, q, 5001, trees.visible([-1], 5001, window, sinks), 64, 128 ** -0.5)
        bound = 2.0 ** -13 * size + 2.0 ** -11 * np.abs(o) + 2.0 ** -24
        for n in (1, 40):
            got = S.window_attention_kv4(torch.from_numpy(np.repeat(q, n, 0)).cuda(), cache,
                                         torch.from_numpy(np.repeat(row[None], n, 0)).cuda(), i32([5001] * n), window, sinks)
            got = got.cpu().numpy().astype(np.float64)
            assert np.all(np.abs(got - o) <= bound)
    assert S.spinq_device_status()[0] == S.SPINQ_OK
