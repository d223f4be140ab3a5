"""spinq_prefix_attention_kv4 on the GPU against attention in 64 bits on the
same codes and scales.

Bar, per value: the weight of a token's codes, p alpha', is rounded to fp16
(2^-11 of it) and meets codes of magnitude at most 8 about the middle code, the
offsets enter in fp32, the output is rounded once (2^-11), the scores carry
fp32 sums (2^-13 of a weight for scores below 64):
|err| <= (2^-11 + 2^-13) sum_t p_t (8 alpha'_t + |beta'_t + 8 alpha'_t|) + 2^-11 |o| + 2^-24."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def _poison(cache, used):
    """NaN scales and codes 0xFF in every slot that is not used."""
    P = cache.k_codes.shape[2]
    free = np.setdiff1d(np.arange(cache.k_codes.shape[0] * P), used)
    page, at = torch.from_numpy(free // P).cuda(), torch.from_numpy(free % P).cuda()
    cache.scales[page, :, at] = float("nan")
    cache.k_codes[page, :, at] = 0xFF
    cache.v_codes[page, :, at] = 0xFF


def _run(S, prefix, lens, Hq, Hkv, D, P, seed=0, spread=1.5, wide=0, v_scale=1.0, scale=None, check=None, stream=None):
    rng = np.random.default_rng(seed)
    tables, pages = ku.page_tables(rng, [prefix] + lens, P)
    cache = ku.random_cache(S, rng, pages, P, Hkv, D)
    cache.scales[..., 2:] *= v_scale
    slots = [ku.token_slots(tables[b], P, 0, n) for b, n in enumerate([prefix] + lens)]
    _poison(cache, np.concatenate(slots))
    B = len(lens)
    width = max(1, max(-(-n // P) for n in lens)) + wide
    table = np.full((B, width), -1, np.int32)
    table[:, :min(width, tables.shape[1])] = tables[1:, :width]
    ptab = tables[0, :max(1, -(-prefix // P))].copy()
    q = (rng.standard_normal((B, Hq, D)) * spread).astype(np.float16)
    dev = lambda a: torch.from_numpy(a).cuda()   # noqa: E731
    args = (dev(q), cache, dev(ptab), prefix, dev(table), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    out = S.prefix_attention_kv4(*args, scale=scale, stream=stream)
    torch.cuda.synchronize()
    sc = 1 / np.sqrt(D) if scale is None else scale
    got = out.cpu().numpy().astype(np.float64)
    pk, pv = ku.slot_values(cache, slots[0])
    for b in (range(B) if check is None else check):
        parts = ku.slot_values(cache, slots[b + 1])
        (uk, ak, bk), (uv, av, bv) = (tuple(np.concatenate([x, y]) for x, y in zip(p, s)) for p, s in zip((pk, pv), parts))
        k, v = uk * ak[..., None] + bk[..., None], uv * av[..., None] + bv[..., None]
        mag = np.broadcast_to((8 * av + np.abs(bv + 8 * av))[..., None], v.shape)
        x = q[b:b + 1].astype(np.float64)
        ref, _ = ku.attention(x, k, v, sc)
        size, _ = ku.attention(x, k, mag, sc)
        err = np.abs(got[b:b + 1] - ref)
        bar = (2.0 ** -11 + 2.0 ** -13) * size + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24
        assert np.all(err <= bar), (b, float((err - bar).max()))
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    return args, out


@pytest.mark.parametrize("prefix,lens,Hq,Hkv,D,P", [
    (1, [0], 8, 8, 128, 16),
    (0, [1, 0, 5], 8, 2, 128, 16),
    (0, [0, 0], 8, 2, 64, 32),
    (37, [0, 3, 200], 32, 8, 128, 64),
    (128, [1], 8, 8, 64, 32),
    (129, [16, 17], 4, 4, 128, 128),
    (1000, [77, 1, 0, 33], 32, 8, 128, 16),
    (700, [300] * 5, 16, 2, 64, 256),
    (500, [9, 600], 24, 8, 128, 16),
    (500, [9, 60, 2], 20, 4, 128, 32),
    (300, [31] * 3, 12, 1, 64, 64),
    (257, [40] * 3, 33, 1, 128, 64),
    (90, [5, 6], 128, 1, 128, 16),
    (2000, [3] * 70, 8, 2, 128, 64),
])
def test_matches_64_bits(S, prefix, lens, Hq, Hkv, D, P):
    _run(S, prefix, lens, Hq, Hkv, D, P, seed=prefix + Hq)


@pytest.mark.parametrize("v_scale", [1e-6, 100.0])
def test_value_scales_far_from_one(S, v_scale):
    """Weights p alpha' keep their 11 bits whatever the values' magnitude."""
    rng = np.random.default_rng(0)
    args, out = None, None
    prefix, lens, Hq, Hkv, D, P = 400, [90, 3], 8, 2, 128, 32
    tables, pages = ku.page_tables(rng, [prefix] + lens, P)
    base = ku.random_cache(S, rng, pages, P, Hkv, D)
    q = torch.from_numpy((rng.standard_normal((2, Hq, D)) * 2).astype(np.float16)).cuda()
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    rest = (dev(tables[0, :13]), prefix, dev(tables[1:, :3]), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    base.scales[..., 2:] *= v_scale
    out = S.prefix_attention_kv4(q, base, *rest)
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    for b in range(2):
        s = np.concatenate([ku.token_slots(tables[0], P, 0, prefix), ku.token_slots(tables[b + 1], P, 0, lens[b])])
        (uk, ak, bk), (uv, av, bv) = ku.slot_values(base, s)
        x = q[b:b + 1].double().cpu().numpy()
        k = uk * ak[..., None] + bk[..., None]
        ref, _ = ku.attention(x, k, uv * av[..., None] + bv[..., None], 1 / np.sqrt(D))
        size, _ = ku.attention(x, k, np.broadcast_to((8 * av + np.abs(bv + 8 * av))[..., None], uv.shape), 1 / np.sqrt(D))
        # fp16 outputs near zero have steps of 2^-24
        bar = (2.0 ** -11 + 2.0 ** -13) * size + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24
        assert np.all(np.abs(got[b:b + 1] - ref) <= bar)


def test_scores_of_every_size(S):
    _run(S, 3000, [500, 0], 8, 2, 128, 64, spread=10.0)
    _run(S, 300, [50, 2], 8, 2, 64, 16, scale=0.0)
    _run(S, 300, [50, 2], 8, 2, 128, 16, scale=-0.1)


def test_long_prefix_and_wide_tables(S):
    _run(S, 20011, [5, 0, 700], 8, 2, 128, 256, wide=9)
    _run(S, 64, [3, 4000], 16, 16, 64, 32)


def test_many_sequences(S):
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 90, 200).tolist()
    _run(S, 1111, lens, 8, 1, 128, 32, check=[0, 57, 128, 199])


def test_agrees_with_the_unpaged_cache(S):
    """A cache [B][S] written by spinq_rotate_quant_kv, its tokens laid into pages."""
    rng = np.random.default_rng(8)
    B, n, Hq, Hkv, D, P = 2, 128, 8, 2, 128, 32
    q, k, v = (torch.from_numpy(rng.standard_normal((B, n, h, D)).astype(np.float16)).cuda() for h in (Hq, Hkv, Hkv))
    kv = S.rotate_quant_kv(q, k, v)
    dense = S.decode_attention_kv4(kv.q_out[:, -1].contiguous(), kv)
    lay = lambda c: c.unflatten(1, (n // P, P)).transpose(2, 3).flatten(0, 1).contiguous()   # noqa: E731
    sc = torch.stack([kv.k_scale, kv.k_zero, kv.v_scale, kv.v_zero], -1)
    cache = S.KV4Pages(lay(kv.k_codes), lay(kv.v_codes), lay(sc))
    table = torch.arange(B * n // P, dtype=torch.int32, device="cuda").view(B, -1)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    paged = S.prefix_attention_kv4(kv.q_out[:, -1].contiguous(), cache, none, 0, table,
                                   torch.full((B,), n, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert (dense.float() - paged.float()).abs().max() <= 4e-3 * dense.float().abs().max()


def test_same_result_every_time_on_any_stream_and_in_a_graph(S):
    args, first = _run(S, 1500, [100, 3, 0, 40], 32, 8, 128, 64, seed=3)
    other = torch.cuda.Stream()
    second = S.prefix_attention_kv4(*args, stream=other)
    torch.cuda.synchronize()
    third = torch.zeros_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.prefix_attention_kv4(*args, out=third)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, second) and torch.equal(first, third)


def test_lengths_are_clamped_to_the_table(S):
    args, _ = _run(S, 40, [20, 31], 8, 2, 128, 16, seed=4)
    q, cache, ptab, prefix, table, lens = args
    cache.scales.nan_to_num_(0.0)
    full = torch.full_like(lens, table.shape[1] * 16)
    table = table.clamp(min=0)
    a = S.prefix_attention_kv4(q, cache, ptab, prefix, table, full)
    b = S.prefix_attention_kv4(q, cache, ptab, prefix, table, full + 1000)
    c = S.prefix_attention_kv4(q, cache, ptab, prefix, table, full * 0 - 5)
    d = S.prefix_attention_kv4(q, cache, ptab, prefix, table, full * 0)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(c, d)


@pytest.mark.parametrize("prefix,lens", [(300, [0, 20, 5]), (0, [9, 20, 5]), (300, [3000, 20, 9000])])
def test_a_query_that_is_not_a_number_gives_its_own_row_only(S, prefix, lens):
    args, _ = _run(S, prefix, lens, 8, 2, 128, 16, seed=6)
    q = args[0].clone()
    clean = S.prefix_attention_kv4(*args)
    q[0, 3, 5] = float("nan")
    out = S.prefix_attention_kv4(q, *args[1:])
    torch.cuda.synchronize()
    bad = torch.zeros(3, 8, dtype=torch.bool, device="cuda")
    bad[0, 3] = True
    assert out[0, 3].isnan().all() and torch.equal(out[~bad], clean[~bad])


def test_many_sequences_beside_a_short_prefix(S):
    """Few SMs have a part of the prefix, the own tokens many CTAs."""
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 60, 160).tolist()
    _run(S, 300, lens, 8, 8, 64, 16, check=[0, 1, 80, 159])
    _run(S, 300, lens, 8, 8, 128, 16, check=[0, 1, 80, 159])


@pytest.mark.parametrize("B,prefix", [(160, 700), (3, 700), (5, 0)])
def test_tokens_appended_just_before_are_seen(S, B, prefix):
    """Append and attention back to back, and with everything finished between them."""
    rng = np.random.default_rng(10)
    Hkv, D, P, own = 8, 128, 16, 64
    pages = -(-prefix // P) + B * own // P
    cache = ku.random_cache(S, rng, pages, P, Hkv, D, poison=False)
    order = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    table, shared = order[:B * own // P].view(B, -1).contiguous(), order[B * own // P:].contiguous()
    if prefix == 0:
        shared = torch.zeros(1, dtype=torch.int32, device="cuda")
    T = B * 16   # 16 new tokens per sequence, at positions 48 .. 63
    slots = (table[:, 3].long()[:, None] * P + torch.arange(P, device="cuda")).flatten()
    lens = torch.full((B,), own, dtype=torch.int32, device="cuda")
    q = torch.from_numpy(rng.standard_normal((B, 16, D)).astype(np.float16)).cuda()
    new = [[torch.from_numpy(rng.standard_normal((T, Hkv, D)).astype(np.float16)).cuda() for _ in range(2)] for _ in range(4)]
    want = []
    for k, v in new:
        S.kv4_append(None, k, v, cache, slots)
        torch.cuda.synchronize()
        want.append(S.prefix_attention_kv4(q, cache, shared, prefix, table, lens))
        torch.cuda.synchronize()
    got = []
    for k, v in new:
        S.kv4_append(None, k, v, cache, slots)
        got.append(S.prefix_attention_kv4(q, cache, shared, prefix, table, lens))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not torch.equal(want[0], want[1])
