"""spinq_prefix_attention_kv4 with queries near fp16's smallest numbers and a scale
that makes their scores ordinary, against attention in 64 bits.

The query values enter the products as they are, so the bar is that of ordinary ones:
|err| <= (2^-11 + 2^-13) sum_t p_t (8 alpha'_t + |beta'_t + 8 alpha'_t|) + 2^-11 |o| + 2^-24."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix,lens", [(0, [3, 40, 200]), (200, [0, 2])])
@pytest.mark.parametrize("D,Hq", [(64, 4), (128, 4), (128, 32)])
@pytest.mark.parametrize("size", [2.0 ** -10, 2.0 ** -14, 2.0 ** -18])
def test_small_queries(prefix, lens, D, Hq, size):
    from paper_2405_16406_gb300 import spinq as S
    rng = np.random.default_rng(int(-np.log2(size)))
    Hkv, P = 2, 16
    tables, pages = ku.page_tables(rng, [prefix] + lens, P)
    cache = ku.random_cache(S, rng, pages, P, Hkv, D)
    q = (rng.standard_normal((len(lens), Hq, D)) * size).astype(np.float16)
    scale = 1 / (size * np.sqrt(D))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()   # noqa: E731
    out = S.prefix_attention_kv4(dev(q), cache, dev(tables[0, :max(1, -(-prefix // P))]), prefix, dev(np.maximum(tables[1:], 0)),
                                 torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=scale)
    torch.cuda.synchronize()
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    got = out.cpu().numpy().astype(np.float64)
    for b in range(len(lens)):
        slots = np.concatenate([ku.token_slots(tables[0], P, 0, prefix), ku.token_slots(tables[b + 1], P, 0, lens[b])])
        (uk, ak, bk), (uv, av, bv) = ku.slot_values(cache, slots)
        k, v = uk * ak[..., None] + bk[..., None], uv * av[..., None] + bv[..., None]
        mag = np.broadcast_to((8 * av + np.abs(bv + 8 * av))[..., None], v.shape)
        x = q[b:b + 1].astype(np.float64)
        ref, mass = ku.attention(x, k, v, scale)[0], ku.attention(x, k, mag, scale)[0]
        err = np.abs(got[b:b + 1] - ref)
        bar = (2.0 ** -11 + 2.0 ** -13) * mass + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24
        assert np.all(err <= bar), (b, float((err / bar).max()))
