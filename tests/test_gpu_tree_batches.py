"""Tree and window attention of batches in which the work is dealt unevenly: one long
sequence among many short ones (cut into more parts than any job of an even batch),
and more sequences than the kernels have threads (the attention kernels and the join
find the same runs with different numbers of sequences per thread).  Inputs and reference
as in test_gpu_tree_attention.py.

Bar: what that file holds for scores, weights and the output, and for values near 0 (a row of one
token whose code all but cancels its offset): the kernels sum p alpha (u - 8) and p alpha (8 + beta /
alpha), whose rounding is relative to 8 alpha and beta and not to the value.  The weights' two parts
are off by 2^-22, the reciprocal of alpha by 2^-23, 8 + beta / alpha by 2^-24 of 8 and of
itself, sums by a few 2^-24: below 2^-21 of sum p (8 alpha + |beta|) in all.  alpha is at most 0.4 here and |beta|
at most 7.5 alpha + 1.7 (normal draws of 0.3): 2^-21 (3.2 + 4.7) < 2^-18."""
import numpy as np
import pytest
import torch

import kv4_util as ku
import test_gpu_tree_attention as trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


_bar = trees._bar


@pytest.fixture(autouse=True)
def bar(monkeypatch):
    monkeypatch.setattr(trees, "_bar", lambda o, size: _bar(o, size) + 2.0 ** -18)


# (1 .. 4 rows, 8 and 16 rows, and 32, 64 and 128 rows on tcgen05; D 64: 32 rows in two jobs)
@pytest.mark.parametrize("nodes,Hq,D", [(1, 1, 128), (1, 4, 128), (2, 4, 128), (4, 4, 128), (8, 4, 128), (16, 4, 128),
                                        (40, 4, 128), (1, 4, 64), (8, 4, 64), (12, 4, 64)])
@pytest.mark.parametrize("ctx", [[30000] + [10] * 39, [10] * 20 + [20000] + [0] * 60 + [9000, 3], [12000] + [1] * 700])
def test_one_long_sequence_among_short_ones(S, ctx, nodes, Hq, D):
    rng = np.random.default_rng(nodes + D)
    trees.run_tree(S, ctx, [trees.forest(rng, nodes if n > 100 else int(rng.integers(0, 2))) for n in ctx], Hq, 1, D, 64,
                   seed=nodes)


@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
@pytest.mark.parametrize("most,Hq,Hkv,D", [(2, 2, 1, 64), (3, 4, 1, 128), (12, 2, 2, 128), (20, 2, 1, 128), (30, 4, 1, 64)])
@pytest.mark.parametrize("B", [129, 257, 300, 513, 700])
def test_more_sequences_than_threads(S, B, most, Hq, Hkv, D, window, sinks):
    """Some without tokens, some without queries."""
    rng = np.random.default_rng(B + most)
    nodes = np.where(rng.random(B) < 0.2, 0, rng.integers(1, most + 1, B))
    nodes[B // 2] = most
    ctx = np.where(rng.random(B) < 0.2, 0, rng.integers(1, 150, B))
    trees.run_tree(S, ctx.tolist(), [trees.forest(rng, int(n)) for n in nodes], Hq, Hkv, D, 16, window, sinks, seed=B)


def test_one_query_each_of_many_sequences(S):
    rng = np.random.default_rng(3)
    for B, top in ((3000, 40), (5000, 9)):
        lens = rng.integers(0, top, B).tolist()
        rows, cache, table, _ = trees.build(S, lens, 1, 64, 16, B)
        q = rows.standard_normal((B, 2, 64)).astype(np.float16)
        dev = lambda x: torch.from_numpy(x).cuda()   # noqa: E731
        got = S.window_attention_kv4(dev(q), cache, dev(table), dev(np.array(lens, np.int32))).cpu().numpy().astype(np.float64)
        (k, ka, kb), (v, va, vb) = ku.slot_values(cache, np.arange(cache.scales.shape[0] * 16))
        k, v = k * ka[..., None] + kb[..., None], v * va[..., None] + vb[..., None]
        for b, n in enumerate(lens):
            at = ku.token_slots(table[b], 16, 0, n)
            o, size = ku.attention(q[b:b + 1].astype(np.float64), k[at], v[at], 1 / 8)
            assert np.all(np.abs(got[b] - o[0]) <= trees._bar(o[0], size[0])), b
    assert S.spinq_device_status()[0] == S.SPINQ_OK
