"""spinq_kv4_plan with numbers that are out of range, free lists that are too short and
depths in each of its forms (one CTA up to 1024 numbers, a cluster up to 8192 tokens, the
tokens over the whole GPU): equal to the same step taken one sequence, one page and one
token at a time, and nothing around the arrays is written."""
import numpy as np
import pytest
import torch

from test_gpu_kv4_plan import OnGpu, Server, pages_of

pytestmark = pytest.mark.gpu

BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


class Clamped(Server):
    """A Server whose numbers may be out of range: lengths and the count are clamped, and freed pages for which the
    list has no room are lost, the last ones first."""

    def step(self, drop, add, total, depths=None, offset=0):
        P, cap = self.P, self.W * self.P
        lens = [min(max(n, 0), cap) for n in self.lens]
        drop = [0] * len(lens) if drop is None else [max(x, 0) for x in drop]
        starts = [max(n - x, 0) for n, x in zip(lens, drop)]
        freed = [int(self.table[b, i]) for b, (s, n) in enumerate(zip(starts, lens)) for i in range(pages_of(s, P), pages_of(n, P))]
        self.stack += freed[:self.capacity - len(self.stack)][::-1]
        self.lens = starts
        if add is None or sum(max(x, 0) for x in add) < 1 << 20:
            return super().step(None, add, total, depths, offset)
        # sums past every array: what the step would do with the first sequences, up to the one that does not fit
        cu = np.cumsum([0] + [max(x, 0) for x in add])
        first = int(np.argmax(cu[1:] > total))
        cut = [x if b < first else 0 for b, x in enumerate(add)]
        want = super().step(None, cut, total, depths, offset)
        granted = [g if b < first or add[b] <= 0 else 0 for b, g in enumerate(want[3])]
        pos = list(want[1])
        for t in range(int(cu[first]), total):   # rows of the sequence that does not fit: positions, no slots
            p = starts[first] + (t - int(cu[first]) if depths is None else int(depths[t])) + offset
            pos[t] = min(max(p, 0), BIG)
        return [min(int(x), total) for x in cu], pos, want[2], granted


def guarded(values, dtype=torch.int32):
    x = torch.full((64 + len(values) + 64,), -77, dtype=dtype, device="cuda")
    x[64:-64] = torch.tensor(values, dtype=dtype, device="cuda")
    return x, x[64:-64]


class GuardedGpu(OnGpu):
    """The arrays with guards around them."""

    def __init__(self, S, host, count=None):
        super().__init__(S, host)
        self.guards = []
        B, W = host.table.shape
        self.lens = self._guard(host.lens)
        self.table = self._guard(host.table.ravel().tolist()).view(B, W)
        self.free = self._guard(self.free.tolist())
        self.count = self._guard([len(host.stack) if count is None else count])

    def _guard(self, values, dtype=torch.int32):
        whole, inner = guarded(values, dtype)
        self.guards.append(whole)
        return inner

    def step(self, drop, add, total, depths=None, offset=0):
        B = len(self.lens)
        plan = self.S.KV4Plan(self._guard([5] * (B + 1)), self._guard([5] * total), self._guard([5] * total, torch.int64),
                              self._guard([5] * B))
        return super().step(drop, add, total, depths, offset, plan=plan)

    def check(self, host, plan, want):
        super().check(host, plan, want)
        for x in self.guards:
            assert (x[:64] == -77).all() and (x[-64:] == -77).all()


FORMS = [(3, 0), (200, 0), (3, 2000), (700, 0), (3, 10000), (700, 10000), (4096, 9000)]   # sequences, rows behind the last


@pytest.mark.parametrize("B,padding", FORMS)
@pytest.mark.parametrize("capacity", [0, 1, 7, 100])
def test_lists_too_short_for_what_is_freed(S, B, padding, capacity):
    rng = np.random.default_rng(B + capacity)
    host = Clamped(rng.integers(0, 70, B).tolist(), 6, 16, 0, seed=B)
    host.stack, host.capacity = [900000 + i for i in range(capacity // 2)], capacity
    gpu = GuardedGpu(S, host)
    for k in range(3):
        drop, add = rng.integers(-1, 90, B).tolist(), rng.integers(-1, 4, B).tolist()
        total = sum(max(x, 0) for x in add) + padding
        want = host.step(drop, add, total)
        gpu.check(host, gpu.step(drop, add, total), want)


@pytest.mark.parametrize("B,padding", FORMS)
def test_counts_and_lengths_out_of_range(S, B, padding):
    rng = np.random.default_rng(B)
    for count in (-5, 3, 40, BIG, -BIG):
        host = Clamped(rng.integers(0, 97, B).tolist(), 6, 16, 30, seed=B)
        host.stack = host.stack + [7000000 + i for i in range(40 - len(host.stack))]
        host.capacity = len(host.stack)
        gpu = GuardedGpu(S, host, count)
        host.stack = host.stack[:min(max(count, 0), host.capacity)]
        wild = rng.choice([-7, -BIG - 1, 97, 5000, BIG], B)
        lens = np.where(rng.random(B) < 0.3, wild, host.lens)
        for b, n in enumerate(lens):   # (lengths past the row: every entry of it is a page)
            host.table[b, :pages_of(min(max(int(n), 0), 96), 16)] = 100 * b + np.arange(pages_of(min(max(int(n), 0), 96), 16))
        host.lens = lens.tolist()
        gpu.lens.copy_(torch.tensor(host.lens, dtype=torch.int32))
        gpu.table.copy_(torch.from_numpy(host.table))
        drop = np.where(rng.random(B) < 0.3, rng.choice([BIG, -BIG - 1, 10 ** 6], B), rng.integers(0, 60, B)).tolist()
        add = np.where(rng.random(B) < 0.2, -BIG - 1, rng.integers(0, 3, B)).tolist()
        total = sum(max(x, 0) for x in add) + padding
        want = host.step(drop, add, total)
        gpu.check(host, gpu.step(drop, add, total), want)


@pytest.mark.parametrize("B,total", [(3, 50), (200, 100), (30, 3000), (700, 500), (30, 10000), (4096, 9000)])
def test_sums_past_every_array(S, B, total):
    """Additions whose sum passes 2^31, from some sequence on."""
    rng = np.random.default_rng(B + total)
    host = Clamped([0] * B, 6, 16, 60, seed=B)
    gpu = GuardedGpu(S, host)
    add = rng.integers(0, 3, B)
    add[B // 2:] = BIG
    add[-1] = 0
    want = host.step(None, add.tolist(), total)
    gpu.check(host, gpu.step(None, add.tolist(), total), want)


@pytest.mark.parametrize("B,padding", FORMS)
@pytest.mark.parametrize("offset", [0, -40, 1000, BIG - 30, -BIG - 1])
def test_depths(S, B, padding, offset):
    rng = np.random.default_rng(B)
    host = Clamped(rng.integers(0, 70, B).tolist(), 6, 16, B + 20, seed=B)
    gpu = GuardedGpu(S, host)
    add = rng.integers(0, 9, B)
    total = int(add.sum()) + padding
    depths = rng.integers(0, 9, total)
    depths[rng.integers(0, total, 1 + total // 20)] = rng.choice([BIG, -BIG - 1, -3], 1 + total // 20)
    args = rng.integers(0, 20, B).tolist(), add.tolist(), total, depths.tolist(), offset
    want = host.step(*args)
    gpu.check(host, gpu.step(*args), want)


@pytest.mark.parametrize("total", [20, 3000, 9000])
def test_tables_without_columns_and_lists_without_room(S, total):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    lens, count = i32([5, 9]), i32([3])
    plan = S.kv4_plan(lens, i32([0, 4]), torch.zeros((2, 0), dtype=torch.int32, device="cuda"), i32([]), count, 16, total,
                      drop=i32([1, 1]))
    torch.cuda.synchronize()
    assert lens.tolist() == [0, 0] and count.item() == 0 and plan.granted.tolist() == [1, 0]
    assert (plan.slots == -1).all() and plan.cu_tokens.tolist() == [0, 0, 4]
