"""spinq_prefix_attention_kv4 where the values' scales alpha' differ between
tokens, against attention in 64 bits on the same codes and scales.

Bar, per value, as where the scales are alike: a token's weight w, proportional
to p alpha', is rounded to fp16 (2^-11 of it) and meets codes of magnitude at most 8
about the middle code, the offsets enter in fp32, the output is rounded once
(2^-11), the scores carry fp32 sums (2^-13 of a weight for scores below 64):
|err| <= (2^-11 + 2^-13) sum_t p_t (8 alpha'_t + |beta'_t + 8 alpha'_t|) + 2^-11 |o| + 2^-24."""
import numpy as np
import pytest
import torch

import kv4_util as ku

pytestmark = pytest.mark.gpu

Hq, Hkv, D, P = 8, 2, 128, 32


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def _outputs(S, rng, prefix, lens, score, alpha, beta=None, scale=None, codes=None, k_alpha=0.02):
    """Outputs, the 64-bit outputs and sum p (8 alpha' + |beta' + 8 alpha'|).  score(n), alpha(n), and
    beta(n, alpha) and codes(n): numbers of n tokens of the prefix or of a sequence, in their order.
    A token's score is about score(n) (queries are positive, a key's offset sets it)."""
    lists = [prefix] + list(lens)
    tables, pages = ku.page_tables(rng, lists, P)
    cache = ku.random_cache(S, rng, pages, P, Hkv, D)
    q = np.abs(rng.standard_normal((len(lens), Hq, D))).astype(np.float16)
    per_beta = D ** 0.5 * (2 / np.pi) ** 0.5   # scale sum_d q_d, on average
    sc, vc = cache.scales.cpu().numpy(), cache.v_codes.cpu().numpy()
    for b, n in enumerate(lists):
        slots = ku.token_slots(tables[b], P, 0, n)
        page, at = slots // P, slots % P
        a = np.broadcast_to(np.asarray(alpha(n), np.float32), n)
        sc[page, :, at, 0] = k_alpha
        sc[page, :, at, 1] = (score(n) / per_beta - 7.5 * k_alpha)[:, None]
        sc[page, :, at, 2] = a[:, None]
        sc[page, :, at, 3] = (-7.5 * a if beta is None else np.asarray(beta(n, a), np.float32))[:, None]
        if codes is not None:
            vc[page, :, at] = codes(n)
    cache.scales.copy_(torch.from_numpy(sc))
    cache.v_codes.copy_(torch.from_numpy(vc))
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()   # noqa: E731
    out = S.prefix_attention_kv4(dev(q), cache, dev(tables[0, :max(1, -(-prefix // P))]), prefix, dev(np.maximum(tables[1:], 0)),
                                 torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=scale)
    torch.cuda.synchronize()
    assert S.spinq_device_status()[0] == S.SPINQ_OK
    got = out.cpu().numpy().astype(np.float64)
    ref, size = np.zeros_like(got), np.zeros_like(got)
    for b in range(len(lens)):
        slots = np.concatenate([ku.token_slots(tables[0], P, 0, prefix), ku.token_slots(tables[b + 1], P, 0, lens[b])])
        (uk, ak, bk), (uv, av, bv) = ku.slot_values(cache, slots)
        k, v = uk * ak[..., None] + bk[..., None], uv * av[..., None] + bv[..., None]
        mag = np.broadcast_to((8 * av + np.abs(bv + 8 * av))[..., None], v.shape)
        x, sm = q[b:b + 1].astype(np.float64), D ** -0.5 if scale is None else scale
        ref[b], size[b] = ku.attention(x, k, v, sm)[0][0], ku.attention(x, k, mag, sm)[0][0]
    return got, ref, size


def _check(got, ref, size, weight=2.0 ** -11 + 2.0 ** -13):
    bar = weight * size + 2.0 ** -11 * np.abs(ref) + 2.0 ** -24
    err = np.abs(got - ref)
    assert np.all(err <= bar), (float((err / bar).max()), np.unravel_index(np.argmax(err / bar), err.shape))


# one tile of rows (two parts of each weight), more than one (one part), own tokens alone and behind a prefix
SHAPES = [(300, [40, 7, 0]), (0, [300, 17]), (1500, [20] * 40), (129, [520, 3])]


@pytest.mark.parametrize("small", [1e-2, 1e-4, 1e-6])
@pytest.mark.parametrize("prefix,lens", SHAPES)
@pytest.mark.parametrize("where", ["first", "last", "spread"])
def test_large_values_without_weight_leave_the_others_their_bits(S, prefix, lens, small, where):
    """A few tokens whose values are 1 / small times the others' and whose scores are 25 below them."""
    def far(n):
        i = np.arange(n)
        return {"first": i < 1, "last": i == n - 1, "spread": i % 37 == 5}[where] & (n > 1)
    rng = np.random.default_rng(1)
    _check(*_outputs(S, rng, prefix, lens, lambda n: np.where(far(n), -25.0, rng.standard_normal(n)),
                     lambda n: 500 * np.where(far(n), 1.0, small) * (1 + 0.3 * rng.random(n))))


@pytest.mark.parametrize("factor", [32.0, 1e4, 1 / 32.0, 1e-4])
@pytest.mark.parametrize("step", [16, 64, 128])
@pytest.mark.parametrize("prefix,lens", SHAPES)
def test_scales_that_grow_or_fall_along_the_tokens(S, prefix, lens, factor, step):
    """From token 2 step on the values are `factor` times the earlier ones', and again later (within 1e-5 .. 1e5)."""
    rng = np.random.default_rng(2)
    _check(*_outputs(S, rng, prefix, lens, lambda n: rng.standard_normal(n),
                     lambda n: np.clip(0.1 * factor ** np.minimum(np.arange(n) // (2 * step), 2), 1e-5, 1e2) * (1 + rng.random(n))))


@pytest.mark.parametrize("prefix,lens", SHAPES)
@pytest.mark.parametrize("equal", ["first", "all", "some"])
def test_rows_of_equal_values(S, prefix, lens, equal):
    """Such a row has scale 0 and its offset alone; it weighs like any other."""
    rng = np.random.default_rng(3)

    def alpha(n):
        i = np.arange(n)
        zero = {"first": i < (n + 1) // 2, "all": i >= 0, "some": i % 3 == 0}[equal]
        return np.where(zero, 0.0, 0.3 * (1 + rng.random(n)))
    _check(*_outputs(S, rng, prefix, lens, lambda n: 2 * rng.standard_normal(n), alpha,
                     lambda n, a: -7.5 * a + rng.standard_normal(n)))


@pytest.mark.parametrize("prefix,lens", [(128, [0, 0]), (128, [32, 16]), (0, [64, 32]), (100, [30] * 32)])
def test_second_parts_of_the_weights(S, prefix, lens):
    """The own tokens, and a prefix with one tile of rows, carry their weights to 2^-22.

    Equal scores (scale 0) and tokens in pairs with opposite codes about the middle, whose scales differ by less
    than 2^-9: the outputs are far smaller than what they are sums of.  Bar: the weight's two fp16
    parts 2^-22, 2^x and log2 2^-22 each, 2^-19 for 16 products of 16 tokens summed in fp32, under 2^-18
    in all; weights in one part (2^-12 of each) are far over it."""
    rng = np.random.default_rng(4)

    def codes(n):
        u = rng.integers(1, 16, (n // 2, 1, D))
        u = np.repeat(np.stack([u, 16 - u], 1).reshape(n, 1, D), Hkv, 1)
        return (u[..., 0::2] | (u[..., 1::2] << 4)).astype(np.uint8)

    def alpha(n):
        a = 0.2 * (1 + rng.random((n // 2, 1)))
        return (a * np.concatenate([np.ones_like(a), 1 + 2.0 ** -9 * rng.random(a.shape)], 1)).reshape(n)
    got, ref, size = _outputs(S, rng, prefix, lens, lambda n: np.zeros(n), alpha, lambda n, a: -8 * a, scale=0.0,
                              codes=codes)
    _check(got, ref, size, weight=2.0 ** -18)
