"""spinq_prompt_attention on the GPU against attention in 64 bits.

Bar, per value: the softmax weights are rounded to fp16 for the product with V
(at most 2^-11 of each weight), the output is rounded once to fp16 (2^-11), and
the scores carry fp32 sums and a 2^-22 exponential (under 2^-13 of a weight
for scores below 64): |err| <= (2^-11 + 2^-13) sum_j p_j |v_j| + 2^-11 |o| + 2^-24."""
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


def _run(S, lq, lk, Hq, Hkv, D, causal, seed=0, scale=None, pad=0, spread=1.5, stream=None, slack=0):
    """pad: rows outside every sequence, between the token rows' end and the tensors' end, hold NaN."""
    rng = np.random.default_rng(seed)
    nq, nk = sum(lq), sum(lk)
    x = (rng.standard_normal((nq + pad, Hq, D)) * spread).astype(np.float16)
    k = rng.standard_normal((nk + pad, Hkv, D)).astype(np.float16)
    v = rng.standard_normal((nk + pad, Hkv, D)).astype(np.float16)
    x[nq:], k[nk:], v[nk:] = np.nan, np.nan, np.nan
    cq, ck = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32) for n in (lq, lk))
    dev = lambda a: torch.from_numpy(a).cuda()   # noqa: E731
    out = torch.full((nq + pad, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    S.prompt_attention(dev(x), dev(k), dev(v), dev(cq), dev(ck), max(lq) + slack, max(lk) + slack, causal=causal,
                       scale=scale, out=out, stream=stream)
    torch.cuda.synchronize()
    sc = 1 / np.sqrt(D) if scale is None else scale
    got = out.cpu().numpy().astype(np.float64)
    assert np.all(got[nq:] == 7.0), "rows outside every sequence are not written"
    for b in range(len(lq)):
        a, e, ka, ke = cq[b], cq[b + 1], ck[b], ck[b + 1]
        i, j = np.arange(e - a)[:, None], np.arange(ke - ka)[None]
        seen = j <= i + (ke - ka) - (e - a) if causal else None
        ref, size = ku.attention(x[a:e].astype(np.float64), k[ka:ke].astype(np.float64), v[ka:ke].astype(np.float64), sc,
                                 seen)
        err = np.abs(got[a:e] - ref)
        assert np.all(err <= _bar(ref, size)), (b, float((err - _bar(ref, size)).max()))
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,Hq,Hkv", [
    ([1], [1], 8, 8),
    ([1, 2, 3], [1, 2, 3], 8, 2),
    ([127], [127], 4, 4),
    ([128], [128], 4, 1),
    ([129, 255, 256, 257], [129, 255, 256, 257], 4, 4),
    ([300, 0, 77, 1], [300, 0, 77, 1], 6, 2),
    ([65, 64, 63], [65, 64, 63], 10, 2),
    ([33], [33], 24, 2),
    ([5, 130], [900, 641], 8, 2),
    ([1, 1, 1], [513, 1, 128], 32, 8),
    ([40, 17], [13, 0], 8, 2),
    ([700], [700], 2, 1),
])
def test_matches_64_bits(S, D, causal, lq, lk, Hq, Hkv):
    _run(S, lq, lk, Hq, Hkv, D, causal, seed=sum(lq) + Hq)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_outside_a_sequence_never_reach_a_result(S, D):
    """NaN after the last sequence, and a neighbour sequence that is all NaN."""
    _run(S, [70, 9], [70, 9], 8, 2, D, True, pad=200)
    _run(S, [70, 9], [200, 131], 8, 2, D, False, pad=3)
    rng = np.random.default_rng(1)
    n = [50, 90, 33]
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    t = [rng.standard_normal((sum(n), h, D)).astype(np.float16) for h in (8, 2, 2)]
    dev = lambda a: torch.from_numpy(a).cuda()   # noqa: E731
    clean = S.prompt_attention(*map(dev, t), dev(cu), dev(cu), 90, 90)
    for bad in (np.nan, np.inf, -np.inf):
        for a in t:
            a[50:140] = bad
        dirty = S.prompt_attention(*map(dev, t), dev(cu), dev(cu), 90, 90)
        torch.cuda.synchronize()
        assert torch.equal(clean[:50], dirty[:50]) and torch.equal(clean[140:], dirty[140:])


def test_long_and_large_scores(S):
    _run(S, [1500], [1500], 2, 1, 128, True, spread=12.0)
    _run(S, [3], [9001], 4, 1, 128, True)
    _run(S, [700], [4500], 2, 2, 64, True)
    _run(S, [20, 1], [3000, 40], 8, 8, 128, True, scale=0.0)
    _run(S, [60], [60], 8, 8, 128, True, scale=-0.2)


@pytest.mark.parametrize("Hq,Hkv", [(7, 1), (9, 3), (33, 1), (71, 1), (128, 1), (100, 1)])
def test_head_groups_of_any_size(S, Hq, Hkv):
    _run(S, [37, 4], [50, 4], Hq, Hkv, 64, True, seed=Hq)


def test_lengths_far_under_the_planned_maximum(S):
    _run(S, [3, 40], [3, 40], 8, 2, 128, True, slack=5000)


def test_strided_rows_of_one_projection(S):
    rng = np.random.default_rng(2)
    T, Hq, Hkv, D = 150, 8, 2, 128
    fused = torch.from_numpy(rng.standard_normal((T, (Hq + 2 * Hkv) * D + 24)).astype(np.float16)).cuda()
    q = fused[:, :Hq * D].unflatten(-1, (Hq, D))
    k = fused[:, Hq * D:(Hq + Hkv) * D].unflatten(-1, (Hkv, D))
    v = fused[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(-1, (Hkv, D))
    cu = torch.tensor([0, 100, 150], dtype=torch.int32, device="cuda")
    a = S.prompt_attention(q, k, v, cu, cu, 100, 100)
    b = S.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), cu, cu, 100, 100)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_same_result_every_time_on_any_stream_and_in_a_graph(S):
    rng = np.random.default_rng(3)
    n = [300, 5, 64]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda")
    q, k, v = (torch.from_numpy(rng.standard_normal((sum(n), h, 128)).astype(np.float16)).cuda() for h in (8, 2, 2))
    first = S.prompt_attention(q, k, v, cu, cu, 300, 300)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    second = S.prompt_attention(q, k, v, cu, cu, 300, 300, stream=other)
    torch.cuda.synchronize()
    third = torch.zeros_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.prompt_attention(q, k, v, cu, cu, 300, 300, out=third)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)


def test_no_queries_is_no_launch(S):
    z = torch.zeros((0, 8, 64), dtype=torch.float16, device="cuda")
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert S.prompt_attention(z, z[:, :2], z[:, :2], cu, cu, 0, 0).shape == (0, 8, 64)


def test_a_query_that_is_not_a_number_gives_its_own_row_only(S):
    rng = np.random.default_rng(5)
    cu = torch.tensor([0, 200, 260], dtype=torch.int32, device="cuda")
    q, k, v = (torch.from_numpy(rng.standard_normal((260, h, 128)).astype(np.float16)).cuda() for h in (8, 2, 2))
    clean = S.prompt_attention(q, k, v, cu, cu, 200, 200)
    q[77, 3, 5] = float("nan")
    q[201, 6, 0] = float("inf")
    out = S.prompt_attention(q, k, v, cu, cu, 200, 200)
    torch.cuda.synchronize()
    bad = torch.zeros(260, 8, dtype=torch.bool, device="cuda")
    bad[77, 3] = bad[201, 6] = True
    assert out[77, 3].isnan().all() and torch.equal(out[~bad], clean[~bad])
