"""spinq_window_prompt_attention on the GPU against attention in 64 bits, with
the bar of the prompt kernel: the weights are rounded to fp16 for the product with V
(2^-11 of each), the output once (2^-11), and scores with fp32 sums and a
2^-22 exponential move a weight by less than 2^-13:
|err| <= (2^-11 + 2^-13) sum_j p_j |v_j| + 2^-11 |o| + 2^-24."""
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
    return (2.0 ** -11 + 2.0 ** -13) * size + 2.0 ** -11 * np.abs(o) + 2.0 ** -24


def _inputs(lq, lk, Hq, Hkv, D, seed, spread=1.5):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((sum(lq), Hq, D)) * spread).astype(np.float16)
    k, v = (rng.standard_normal((sum(lk), Hkv, D)).astype(np.float16) for _ in range(2))
    cq, ck = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32) for n in (lq, lk))
    return x, k, v, cq, ck


def _run(S, lq, lk, Hq, Hkv, D, window, sinks, seed=0, scale=None, **kw):
    x, k, v, cq, ck = _inputs(lq, lk, Hq, Hkv, D, seed)
    dev = lambda a: torch.from_numpy(a).cuda()   # noqa: E731
    out = S.window_prompt_attention(dev(x), dev(k), dev(v), dev(cq), dev(ck), max(lq), max(lk), window, sinks, scale=scale, **kw)
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    for b in range(len(lq)):
        a, e, ka, ke = cq[b], cq[b + 1], ck[b], ck[b + 1]
        p, j = np.arange(e - a)[:, None] + (ke - ka) - (e - a), np.arange(ke - ka)[None]
        seen = (j <= p) & ((p - j < window) | (j < sinks))
        ref, size = ku.attention(x[a:e].astype(np.float64), k[ka:ke].astype(np.float64), v[ka:ke].astype(np.float64),
                                 1 / np.sqrt(D) if scale is None else scale, seen)
        err = np.abs(got[a:e] - ref)
        assert np.all(err <= _bar(ref, size)), (b, float((err - _bar(ref, size)).max()))
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (127, 0), (128, 128), (129, 5), (300, 200), (700, 1000)])
@pytest.mark.parametrize("lq,lk,Hq,Hkv", [
    ([1], [1], 8, 8),
    ([129, 255, 256, 257], [129, 255, 256, 257], 4, 4),
    ([300, 0, 77, 1], [300, 0, 77, 1], 6, 2),
    ([5, 130, 1], [900, 641, 1300], 8, 2),
    ([40, 17], [13, 0], 8, 2),
    ([900], [900], 2, 1),
])
def test_matches_64_bits(S, D, window, sinks, lq, lk, Hq, Hkv):
    _run(S, lq, lk, Hq, Hkv, D, window, sinks, seed=sum(lq) + Hq)


@pytest.mark.parametrize("Hq,Hkv", [(7, 1), (33, 1), (71, 1), (128, 1)])
def test_head_groups_of_any_size(S, Hq, Hkv):
    _run(S, [37, 140], [50, 500], Hq, Hkv, 64, 33, 3, seed=Hq)


def test_long(S):
    _run(S, [2500], [2500], 4, 2, 128, 640, 20)
    _run(S, [3], [9001], 4, 1, 128, 4096, 4)
    _run(S, [60], [600], 8, 8, 128, 50, 9, scale=-0.2)
    _run(S, [60], [600], 8, 8, 128, 50, 9, scale=0.0)


@pytest.mark.parametrize("window,sinks", [(1 << 40, 0), (2 ** 31, 7), (2 ** 31 - 1, 0), (700, 0), (1, 1 << 40), (5, 2 ** 31 - 1)])
def test_a_window_over_everything_is_the_causal_prompt(S, window, sinks):
    x, k, v, cq, ck = _inputs([300, 5], [700, 5], 8, 2, 128, 1)
    t = [torch.from_numpy(a).cuda() for a in (x, k, v, cq, ck)]
    a = S.window_prompt_attention(*t, 300, 700, window, sinks)
    b = S.prompt_attention(*t, 300, 700)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_rows_of_other_sequences_never_reach_a_result(S):
    x, k, v, cq, ck = _inputs([50, 90, 33], [150, 190, 533], 8, 2, 64, 2)
    dev = lambda a: torch.from_numpy(a).cuda()   # noqa: E731
    clean = S.window_prompt_attention(*map(dev, (x, k, v, cq, ck)), 90, 533, 40, 3)
    x[50:140] = k[150:340] = v[150:340] = np.nan
    dirty = S.window_prompt_attention(*map(dev, (x, k, v, cq, ck)), 90, 533, 40, 3)
    torch.cuda.synchronize()
    assert torch.equal(clean[:50], dirty[:50]) and torch.equal(clean[140:], dirty[140:])


def test_same_result_on_any_stream_and_in_a_graph(S):
    t = [torch.from_numpy(a).cuda() for a in _inputs([300, 5, 64], [300, 500, 64], 8, 2, 128, 3)]
    first = S.window_prompt_attention(*t, 300, 500, 100, 4)
    torch.cuda.synchronize()
    second = S.window_prompt_attention(*t, 300, 500, 100, 4, stream=torch.cuda.Stream())
    third = torch.full_like(first, 7.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.window_prompt_attention(*t, 300, 500, 100, 4, out=third)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)


def test_rows_behind_the_last_sequence_are_left(S):
    x, k, v, cq, ck = _inputs([70, 30], [70, 230], 8, 2, 128, 4)
    t = [torch.from_numpy(a).cuda() for a in (x, k, v, cq[:2].copy(), ck[:2].copy())]
    out = torch.full((100, 8, 128), 7.0, dtype=torch.float16, device="cuda")
    S.window_prompt_attention(*t, 70, 70, 20, 2, out=out)
    torch.cuda.synchronize()
    assert (out[70:] == 7.0).all() and not (out[:70] == 7.0).all(-1).any()


def test_no_queries_is_no_launch(S):
    z = torch.zeros((0, 8, 64), dtype=torch.float16, device="cuda")
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert S.window_prompt_attention(z, z[:, :2], z[:, :2], cu, cu, 0, 0, 5).shape == (0, 8, 64)
