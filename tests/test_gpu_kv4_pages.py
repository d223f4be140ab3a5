"""The paged 4-bit cache on the GPU: spinq_kv4_append and spinq_kv4_read against
plain 64-bit forms.

Bars.  Codes: as for the unpaged KV path, +-1 on at most 1e-4 of the values
(the rounding of a value that lies between two codes); scales within 1e-5.
The fp32 path from the input to q_out has, per value, the norm (sum of
squares, square root, quotient, two products: under 13 half-ulps), the rotation
(3) and log2 D <= 7 butterfly stages: under 2^-19 of the row's norm, and one
rounding to fp16.  Read-back: one rounding to fp16 of an fp32 fma."""
import numpy as np
import pytest
import torch

import kv4_util as ku
from parity_util import assert_codes_close, assert_scale_close, assert_zero_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def _case(rng, T, Hq, Hkv, D):
    x = rng.standard_normal((T, (Hq + 2 * Hkv) * D)).astype(np.float32)
    x[:, ::37] *= 8   # a few large channels
    return torch.from_numpy(x.astype(np.float16)).cuda()


def _split(x, Hq, Hkv, D):
    a, b = Hq * D, (Hq + Hkv) * D
    return x[:, :a].unflatten(-1, (Hq, D)), x[:, a:b].unflatten(-1, (Hkv, D)), x[:, b:].unflatten(-1, (Hkv, D))


def _ulp16(v):
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -14))) - 10)


@pytest.mark.parametrize("T,Hq,Hkv,D,P,rotary,interleaved,norm,clip", [
    (1, 32, 8, 128, 16, 128, False, True, 1.0),
    (67, 32, 8, 128, 64, 128, True, True, 1.0),
    (67, 24, 8, 128, 32, 64, False, False, 1.0),
    (33, 20, 4, 128, 256, 96, False, True, 0.95),
    (33, 5, 1, 128, 16, 32, True, False, 1.0),
    (41, 8, 8, 64, 32, 64, False, True, 1.0),
    (41, 3, 3, 64, 16, 48, False, False, 0.9),
    (41, 16, 2, 64, 128, 32, True, True, 1.0),
    (29, 8, 2, 128, 64, 0, False, True, 1.0),
    (29, 8, 2, 64, 64, 0, False, False, 1.0),
])
def test_append_matches_64_bits(S, T, Hq, Hkv, D, P, rotary, interleaved, norm, clip):
    rng = np.random.default_rng(T * 1000 + Hq + rotary)
    q, k, v = _split(_case(rng, T, Hq, Hkv, D), Hq, Hkv, D)
    pages = -(-T // P) + 3
    cache = S.kv4_pages(pages, P, Hkv, D)
    cache.k_codes.fill_(0xA5)
    cache.v_codes.fill_(0x5A)
    cache.scales.fill_(float("nan"))
    slots = rng.permutation(pages * P)[:T].astype(np.int64)
    pos = rng.integers(0, 500, T).astype(np.int32)
    table = ku.cos_sin(500, rotary) if rotary else None
    w = [(1 + 0.2 * rng.standard_normal(D)).astype(np.float16) for _ in range(2)] if norm else [None, None]
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()   # noqa: E731
    out = S.kv4_append(q, k, v, cache, dev(slots), dev(pos) if rotary else None, dev(table), dev(w[0]), dev(w[1]), 1e-5,
                       interleaved, clip)
    torch.cuda.synchronize()
    ref_q = ku.rotated_rows(q.cpu().numpy(), w[0], 1e-5, pos, table, interleaved)
    ref_k = ku.rotated_rows(k.cpu().numpy(), w[1], 1e-5, pos, table, interleaved)
    size = np.linalg.norm(ref_q, axis=-1, keepdims=True)
    assert np.all(np.abs(out.cpu().numpy() - ref_q) <= 0.5 * _ulp16(ref_q) * 1.01 + 2.0 ** -19 * size)
    for (u, al, be), y, name in zip(ku.slot_values(cache, slots), (ref_k, v.cpu().numpy().astype(np.float64)), "KV"):
        ru, ra, rb = ku.codes_of(y, clip)
        assert_codes_close(u.reshape(-1, D), ru.reshape(-1, D), name)
        assert_scale_close(al.reshape(-1), ra.reshape(-1), name)
        assert_zero_close(be.reshape(-1), rb.reshape(-1), ra.reshape(-1), name)
    # no other slot is touched
    free = np.setdiff1d(np.arange(pages * P), slots)
    page, at = torch.from_numpy(free // P).cuda(), torch.from_numpy(free % P).cuda()
    assert bool((cache.k_codes[page, :, at] == 0xA5).all()) and bool((cache.v_codes[page, :, at] == 0x5A).all())
    assert bool(torch.isnan(cache.scales[page, :, at]).all())
    assert S.spinq_device_status()[0] == S.SPINQ_OK


@pytest.mark.parametrize("D", [64, 128])
def test_append_agrees_with_the_unpaged_cache(S, D):
    """Without norms and rotation the pages hold what spinq_rotate_quant_kv writes."""
    rng = np.random.default_rng(D)
    T, Hq, Hkv, P = 77, 8, 4, 32
    q, k, v = _split(_case(rng, T, Hq, Hkv, D), Hq, Hkv, D)
    ref = S.rotate_quant_kv(q[None].contiguous(), k[None].contiguous(), v[None].contiguous())
    cache = S.kv4_pages(3, P, Hkv, D)
    slots = torch.arange(T, device="cuda")
    S.kv4_append(q, k, v, cache, slots)
    torch.cuda.synchronize()
    (ku_, ka, _), (vu, va, _) = ku.slot_values(cache, slots.cpu().numpy())
    assert_codes_close(ku_.reshape(-1, D), ku.unpack(ref.k_codes[0].cpu().numpy()).reshape(-1, D), "K")
    assert_codes_close(vu.reshape(-1, D), ku.unpack(ref.v_codes[0].cpu().numpy()).reshape(-1, D), "V")
    assert_scale_close(ka.reshape(-1), ref.k_scale[0].double().cpu().numpy().reshape(-1), "K")
    assert_scale_close(va.reshape(-1), ref.v_scale[0].double().cpu().numpy().reshape(-1), "V")


def test_append_skips_slots_outside_the_cache_and_takes_no_queries(S):
    rng = np.random.default_rng(1)
    T, Hkv, D, P = 9, 2, 128, 16
    _, k, v = _split(_case(rng, T, 2, Hkv, D), 2, Hkv, D)
    cache = S.kv4_pages(1, P, Hkv, D)
    cache.k_codes.fill_(0xA5)
    slots = torch.tensor([3, -1, 16, 5, 1 << 40, -(1 << 50), 0, 17, 15], device="cuda")
    assert S.kv4_append(None, k, v, cache, slots) is None
    torch.cuda.synchronize()
    written = [s for s in slots.tolist() if 0 <= s < P]
    for s in range(P):
        assert bool((cache.k_codes[0, :, s] == 0xA5).all()) == (s not in written)


def test_append_constant_rows_have_zero_scale(S):
    cache = S.kv4_pages(1, 16, 1, 64)
    z = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda")
    S.kv4_append(None, z, z + 3, cache, torch.tensor([0, 1], device="cuda"))
    torch.cuda.synchronize()
    assert cache.scales[0, 0, :2].tolist() == [[0, 0, 0, 3], [0, 0, 0, 3]]
    assert not cache.k_codes[0, 0, :2].any() and not cache.v_codes[0, 0, :2].any()


def test_append_in_place_queries_and_empty(S):
    rng = np.random.default_rng(2)
    T, H, D = 19, 4, 128
    q, k, v = (t.contiguous() for t in _split(_case(rng, T, H, H, D), H, H, D))
    cache = S.kv4_pages(2, 16, H, D)
    slots = torch.arange(T, device="cuda")
    apart = S.kv4_append(q, k, v, cache, slots)
    same = S.kv4_append(q, k, v, cache, slots, q_out=q)
    torch.cuda.synchronize()
    assert same.data_ptr() == q.data_ptr() and torch.equal(apart, same)
    assert S.kv4_append(q[:0], k[:0], v[:0], cache, slots[:0]).shape == (0, H, D)


@pytest.mark.parametrize("lens,starts,Hkv,D,P", [
    ([1], None, 8, 128, 16),
    ([0, 37, 0, 130, 1, 0], None, 8, 128, 64),
    ([77, 5], [13, 90], 3, 64, 32),
    ([300, 257], [0, 255], 1, 128, 256),
    ([45, 63], [16, 1], 5, 64, 16),
])
def test_read_matches_64_bits(S, lens, starts, Hkv, D, P):
    rng = np.random.default_rng(sum(lens))
    ends = [n + (0 if starts is None else starts[b]) for b, n in enumerate(lens)]
    table, pages = ku.page_tables(rng, ends, P)
    cache = ku.random_cache(S, rng, pages, P, Hkv, D)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    k, v = S.kv4_read(cache, torch.from_numpy(table).cuda(), torch.from_numpy(cu).cuda(), int(cu[-1]), starts=st)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        if n == 0:
            continue
        slots = ku.token_slots(table[b], P, 0 if starts is None else starts[b], n)
        for (u, al, be), got in zip(ku.slot_values(cache, slots), (k, v)):
            ref = u * al[..., None] + be[..., None]
            g = got[cu[b]:cu[b + 1]].cpu().numpy().astype(np.float64)
            bar = 0.5 * _ulp16(ref) + 2.0 ** -23 * (15 * al + np.abs(be))[..., None]
            assert np.all(np.abs(g - ref) <= bar)


def test_read_past_the_table_gives_zeros(S):
    rng = np.random.default_rng(3)
    cache = ku.random_cache(S, rng, 2, 16, 2, 64)
    table = torch.tensor([[1], [7], [-3]], dtype=torch.int32, device="cuda")   # the last two name no page
    cu = torch.tensor([0, 20, 22, 24], dtype=torch.int32, device="cuda")
    k, v = S.kv4_read(cache, table, cu, 24)
    torch.cuda.synchronize()
    assert bool(k[:16].any()) and not k[16:].any() and not v[16:].any()


def test_cache_over_four_gigabytes(S):
    """Slots whose byte offsets pass 32 bits, in the codes (4.5 GB each) and the scales."""
    Hkv, D, P = 8, 128, 256
    pages = 36000
    cache = S.kv4_pages(pages, P, Hkv, D)
    assert cache.k_codes.numel() > 1 << 32
    rng = np.random.default_rng(4)
    T = 24
    _, k, v = _split(_case(rng, T, 2, Hkv, D), 2, Hkv, D)
    table = np.array([[pages - 1, 3, pages - 2]], dtype=np.int32)
    slots = ku.token_slots(table[0], P, 2 * P - 12, T)
    S.kv4_append(None, k, v, cache, torch.from_numpy(slots).cuda())
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    ko, vo = S.kv4_read(cache, torch.from_numpy(table).cuda(), cu, T,
                        starts=torch.tensor([2 * P - 12], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for got, x in ((ko, ku.rotated_rows(k.cpu().numpy(), None, 0, None, None, False)),
                   (vo, v.cpu().numpy().astype(np.float64))):
        u, al, be = ku.codes_of(x)
        err = np.abs(got.cpu().numpy() - x)
        assert np.all(err <= 0.5 * al[..., None] + 2e-3 * np.abs(x).max())


def test_append_and_read_on_another_stream_and_in_a_graph(S):
    rng = np.random.default_rng(5)
    T, Hq, Hkv, D = 40, 8, 2, 128
    q, k, v = _split(_case(rng, T, Hq, Hkv, D), Hq, Hkv, D)
    slots = torch.arange(T, device="cuda")
    table = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    cache = S.kv4_pages(3, 16, Hkv, D)
    q0 = S.kv4_append(q, k, v, cache, slots)
    k0, v0 = S.kv4_read(cache, table, cu, T)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    cache.k_codes.zero_(), cache.v_codes.zero_()
    torch.cuda.synchronize()
    q1 = S.kv4_append(q, k, v, cache, slots, stream=other)
    k1, v1 = S.kv4_read(cache, table, cu, T, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(q0, q1) and torch.equal(k0, k1) and torch.equal(v0, v1)
    g = torch.cuda.CUDAGraph()
    q2, k2, v2 = torch.empty_like(q0), torch.empty_like(k0), torch.empty_like(v0)
    with torch.cuda.graph(g):
        S.kv4_append(q, k, v, cache, slots, q_out=q2)
        S.kv4_read(cache, table, cu, T, k=k2, v=v2)
    cache.k_codes.zero_(), cache.v_codes.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(q0, q2) and torch.equal(k0, k2) and torch.equal(v0, v2)
