"""Tree and window attention over tokens whose scales are not numbers, where a
sequence's keys are cut into parts that are joined: such a token may be a part by
itself, fill several parts, or lie in a part whose scores are far below the others'.
A row that sees it is NaN in every value, any other row keeps its bits."""
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


class Case:
    """One sequence of n tokens (and one of 40 beside it, whose rows keep theirs), `nodes` queries each."""

    def __init__(self, S, n, nodes, Hq, Hkv, D, P=64, seed=0):
        rng = np.random.default_rng(seed + n)
        self.S, self.P, self.n, self.nodes, self.G = S, P, n, nodes, Hq // Hkv
        table, pages = ku.page_tables(rng, [n, 40 + nodes], P)
        self.cache = ku.random_cache(S, rng, pages, P, Hkv, D)
        self.rows, self.table = table, torch.from_numpy(table).cuda()
        self.lens, self.cu = i32([n, 40 + nodes]), i32([0, nodes, 2 * nodes])
        self.q = torch.from_numpy(rng.standard_normal((2 * nodes, Hq, D)).astype(np.float16)).cuda()

    def run(self, parents=None, window=0, sinks=0):
        out = self.S.tree_attention_kv4(self.q, self.cache, self.table, self.lens, self.cu, self.nodes,
                                        None if parents is None else i32(parents * 2), window, sinks)
        torch.cuda.synchronize()
        return out

    def scales(self, first, end, heads=slice(None)):
        """The scales of tokens first .. end - 1, to be written."""
        slots = ku.token_slots(self.rows[0], self.P, first, end - first)
        page, at = torch.from_numpy(slots // self.P).cuda(), torch.from_numpy(slots % self.P).cuda()
        return lambda which, x: self.cache.scales[:, heads].transpose(1, 2)[..., which].index_put_((page, at), x)


# few rows with second parts in idle columns, 8 and 16 rows, and 32, 64 and 128 rows on tcgen05
SIZES = [(1, 32, 8, 128), (2, 32, 8, 128), (4, 32, 8, 128), (8, 32, 8, 128), (12, 32, 8, 128), (64, 32, 8, 128),
         (1, 8, 8, 64), (4, 8, 1, 64), (9, 8, 1, 64)]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [257, 513, 769, 1025, 2049, 16001])
@pytest.mark.parametrize("nodes,Hq,Hkv,D", SIZES)
def test_the_last_token(S, nodes, Hq, Hkv, D, n, bad):
    """The last node of a chain, the first token of a unit: only its own rows see it."""
    x = Case(S, n, nodes, Hq, Hkv, D)
    clean = x.run()
    x.scales(n - 1, n)(slice(None), torch.tensor(bad, device="cuda"))
    dirty = x.run()
    assert dirty[nodes - 1].isnan().all()
    rest = [i for i in range(2 * nodes) if i != nodes - 1]
    assert torch.equal(clean[rest], dirty[rest]) and not clean.isnan().any()


@pytest.mark.parametrize("which", [slice(0, 2), slice(2, 4)])
@pytest.mark.parametrize("first,end", [(0, 700), (640, 1408), (1300, 2049), (1, 2)])
@pytest.mark.parametrize("nodes,Hq,Hkv,D", SIZES)
def test_context_tokens_that_fill_parts(S, nodes, Hq, Hkv, D, first, end, which):
    """Keys or values that are not numbers over several units of the context, in one kv head: every row of the
    head's group is NaN, no other."""
    n = 2049 + nodes
    x = Case(S, n, nodes, Hq, Hkv, D)
    clean = x.run()
    head = Hkv - 1
    x.scales(first, end, slice(head, head + 1))(which, torch.tensor(float("nan"), device="cuda"))
    dirty = x.run()
    group = slice(head * x.G, Hq)
    assert dirty[:nodes, group].isnan().all()
    assert torch.equal(dirty[:nodes, :head * x.G], clean[:nodes, :head * x.G]) and torch.equal(dirty[nodes:], clean[nodes:])
    seen_not = x.run(window=2, sinks=0)   # windows that lie behind all of it
    assert not seen_not.isnan().any() or end > 2047


@pytest.mark.parametrize("nodes,Hq,Hkv,D", SIZES)
def test_a_part_far_below_the_others(S, nodes, Hq, Hkv, D):
    """Scores of 1000 tokens are 400 or so below the others': their weights are 0 in 32 bits, a value among them
    that is not a number still makes the sum none."""
    n = 3000 + nodes
    x = Case(S, n, nodes, Hq, Hkv, D)
    x.q.abs_()
    x.scales(1000, 2000)(1, torch.tensor(-5.0 * D ** 0.5, device="cuda"))
    clean = x.run()
    assert not clean.isnan().any()
    x.scales(1500, 1501)(slice(2, 4), torch.tensor(float("nan"), device="cuda"))
    dirty = x.run()
    assert dirty[:nodes].isnan().all() and torch.equal(dirty[nodes:], clean[nodes:])
