"""spinq_kv4_plan and spinq_kv4_keep on the GPU against the same steps taken one
sequence, one page and one token at a time.  Whole numbers: equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


def pages_of(n, P):
    return -(-n // P)


class Server:
    """Lengths, page lists and the stack of free pages, on the host."""

    def __init__(self, lens, W, P, spare, seed=0, capacity=None):
        rng = np.random.default_rng(seed)
        held = [pages_of(n, P) for n in lens]
        N = sum(held) + spare
        order = rng.permutation(N).tolist()
        self.W, self.P, self.lens = W, P, list(lens)
        self.table = np.full((len(lens), W), -7, np.int32)
        for b, n in enumerate(held):
            for i in range(n):
                self.table[b, i] = order.pop()
        self.stack, self.capacity = order, N if capacity is None else capacity

    def step(self, drop, add, total, depths=None, offset=0):
        P, cap = self.P, self.W * self.P
        cu, pos, slots, granted = [0], [0] * total, [-1] * total, []
        freed, starts = [], []
        for b, n in enumerate(self.lens):
            n = min(max(n, 0), cap)
            s = max(n - max(drop[b], 0), 0) if drop is not None else n
            starts.append(s)
            freed += [int(self.table[b, i]) for i in range(pages_of(s, P), pages_of(n, P))]
        self.stack += freed[::-1]
        out_of_pages = False
        for b, s in enumerate(starts):
            n = max(add[b], 0) if add is not None else 0
            fits = n == 0 or (cu[-1] + n <= total and s + n <= cap)
            need = pages_of(s + n, P) - pages_of(s, P) if fits else 0
            if need > 0 and (out_of_pages or need > len(self.stack)):
                out_of_pages, fits = True, False
            granted.append(int(fits))
            if fits:
                for i in range(need):
                    self.table[b, pages_of(s, P) + i] = self.stack.pop()
            for i in range(n):
                t = cu[-1] + i
                if t < total:
                    p = s + (i if depths is None else int(depths[t])) + offset
                    pos[t] = min(max(p, 0), 2 ** 31 - 1)
                    if fits:
                        slots[t] = int(self.table[b, (s + i) // P]) * P + (s + i) % P
            self.lens[b] = s + n if fits else s
            cu.append(cu[-1] + n)
        return [min(x, total) for x in cu], pos, slots, granted


class OnGpu:
    def __init__(self, S, host):
        self.S, self.P = S, host.P
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        self.lens, self.table = i32(host.lens), torch.from_numpy(host.table.copy()).cuda()
        self.free = torch.full((host.capacity,), -9, dtype=torch.int32, device="cuda")
        self.free[:len(host.stack)] = i32(host.stack)
        self.count = i32([len(host.stack)])

    def step(self, drop, add, total, depths=None, offset=0, **kw):
        i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        return self.S.kv4_plan(self.lens, i32(add), self.table, self.free, self.count, self.P, total, drop=i32(drop),
                               depths=i32(depths), position_offset=offset, **kw)

    def check(self, host, plan, want):
        torch.cuda.synchronize()
        for got, x in zip((plan.cu_tokens, plan.positions, plan.slots, plan.granted), want):
            assert got.tolist() == x
        assert self.lens.tolist() == host.lens
        assert np.array_equal(self.table.cpu().numpy(), host.table)
        assert self.count.item() == len(host.stack) and self.free[:len(host.stack)].tolist() == host.stack


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("B,longest,spare,padding", [(1, 1, 5, 0), (1, 900, 40, 3), (8, 3, 4, 0), (7, 300, 20, 50), (33, 40, 2, 7),
                                                    (513, 20, 300, 1), (700, 60, 10, 64), (4096, 2, 2000, 5)])
def test_steps_of_a_server(S, P, B, longest, spare, padding):
    """Random drops and additions, pages running short now and then; the state carries over."""
    rng = np.random.default_rng(B + P)
    W = pages_of(3 * longest + 40, P)
    host = Server(rng.integers(0, 2 * longest + 1, B).tolist(), W, P, spare, seed=B)
    gpu = OnGpu(S, host)
    for k in range(4):
        drop = None if k == 1 else rng.integers(-1, 2 * longest, B).tolist()
        add = None if k == 2 else rng.integers(-1, longest + 1, B).tolist()
        total = sum(max(x, 0) for x in add or [0]) + padding
        want = host.step(drop, add, total, offset=5 * k)
        gpu.check(host, gpu.step(drop, add, total, offset=5 * k), want)
    held = [int(p) for b, n in enumerate(host.lens) for p in host.table[b, :pages_of(n, P)]]
    assert sorted(held + host.stack) == list(range(host.capacity)), "no page lost, none twice"


def test_sequences_that_take_what_they_give_keep_their_pages(S):
    host = Server([100, 33, 16, 1], 10, 16, 7)
    gpu = OnGpu(S, host)
    before = host.table.copy()
    for _ in range(2):
        want = host.step([40, 33, 16, 1], [40, 33, 16, 1], 90)
        gpu.check(host, gpu.step([40, 33, 16, 1], [40, 33, 16, 1], 90), want)
        assert np.array_equal(before, host.table)


def test_rows_that_do_not_fit_are_refused(S):
    """A row of the table too short for one sequence, the tokens' rows for another, pages for a third."""
    host = Server([60, 0, 10, 5, 0], 4, 16, 3)
    gpu = OnGpu(S, host)
    add = [10, 17, 5, 40, 1]
    want = host.step(None, add, 71)   # 60 + 10 > 64; the last token's row is 72
    assert want[3] == [0, 1, 1, 0, 0]
    gpu.check(host, gpu.step(None, add, 71), want)


def test_lengths_of_zero_and_nothing_to_do(S):
    host = Server([0, 0, 0], 2, 16, 4)
    gpu = OnGpu(S, host)
    gpu.check(host, gpu.step(None, None, 0), host.step(None, None, 0))
    gpu.check(host, gpu.step([1, 2, 3], [0, 0, 0], 4), host.step([1, 2, 3], [0, 0, 0], 4))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    count = i32(2)
    plan = S.kv4_plan(i32(), None, torch.zeros((0, 3), dtype=torch.int32, device="cuda"), i32(4, 5), count, 16, 3)
    torch.cuda.synchronize()
    assert plan.cu_tokens.tolist() == [0] and plan.slots.tolist() == [-1] * 3 and plan.positions.tolist() == [0] * 3
    assert count.item() == 2


def test_numbers_out_of_range_stay_in_bounds(S):
    """Lengths below zero and past the row, sums past 2^31, a count that the list cannot have, a list with no
    room for what is freed: guarded memory around every array stays as it is."""
    big = 2 ** 31 - 1
    for lens, drop, add, count, N in (([-5, 1000, 20], [big, 0, -3], [big, big, big], 3, 6), ([64, 64, 64], [64, 64, 64], [1, 2, 3], 99, 4),
                                      ([64, 64, 64], [big, big, big], [-1, 0, 4], -7, 5), ([64, 0, 64], [10, 0, 64], [4, 4, 4], 4, 4)):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        fields = {"lens": lens, "table": list(range(12)), "free": list(range(50, 50 + N)), "count": [count], "cu": [0] * 4,
                  "pos": [0] * 9, "granted": [0] * 3}
        guard = {k: i32([-77] * 64 + v + [-77] * 64) for k, v in fields.items()}
        at = {k: guard[k][64:-64] for k in fields}
        slots = torch.full((64 + 9 + 64,), -77, dtype=torch.int64, device="cuda")
        plan = S.KV4Plan(at["cu"], at["pos"], slots[64:-64], at["granted"])
        S.kv4_plan(at["lens"], i32(add), at["table"].view(3, 4), at["free"], at["count"], 16, 9, drop=i32(drop), plan=plan)
        torch.cuda.synchronize()
        for g in list(guard.values()) + [slots]:
            assert (g[:64] == -77).all() and (g[-64:] == -77).all()
        assert 0 <= at["count"].item() <= N
        assert all(0 <= n <= 64 for n in at["lens"].tolist())


def test_depths_are_positions_of_a_tree(S):
    host = Server([20, 31], 6, 16, 8)
    gpu = OnGpu(S, host)
    depths = [0, 1, 1, 2, 0, 1, 99]
    want = host.step([2, 0], [4, 2], 7, depths=depths, offset=1000)
    assert want[1] == [1018, 1019, 1019, 1020, 1031, 1032, 0]
    gpu.check(host, gpu.step([2, 0], [4, 2], 7, depths=depths, offset=1000), want)


def test_steps_replay_from_a_graph_and_run_on_any_stream(S):
    host = Server([5, 40, 100, 0], 16, 16, 30)
    gpu = OnGpu(S, host)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    add, drop = i32([1, 1, 1, 1]), i32([0, 0, 0, 0])
    empty = lambda n, t: torch.zeros(n, dtype=t, device="cuda")   # noqa: E731
    plan = S.KV4Plan(empty(5, torch.int32), empty(70, torch.int32), empty(70, torch.int64), empty(4, torch.int32))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.kv4_plan(gpu.lens, add, gpu.table, gpu.free, gpu.count, 16, 70, drop=drop, plan=plan)
    for d, a in (([0, 0, 0, 0], [1, 1, 1, 1]), ([3, 0, 100, 0], [20, 9, 40, 1]), ([0, 50, 0, 0], [0, 0, 33, 2])):
        add.copy_(i32(a))
        drop.copy_(i32(d))
        g.replay()
        gpu.check(host, plan, host.step(d, a, 70))
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = gpu.step([1, 1, 1, 1], [2, 0, 2, 0], 4, stream=other)
    gpu.check(host, plan, host.step([1, 1, 1, 1], [2, 0, 2, 0], 4))


# ------------------------------------------------------------------ keep
def _cache(S, rng, pages, P, Hkv, D):
    r = lambda hi, *s: torch.from_numpy(rng.integers(0, hi, s).astype(np.uint8)).cuda()   # noqa: E731
    scales = torch.from_numpy(rng.standard_normal((pages, Hkv, P, 4)).astype(np.float32)).cuda()
    return S.KV4Pages(r(256, pages, Hkv, P, D // 2), r(256, pages, Hkv, P, D // 2), scales)


def _copy(cache):
    return [x.clone() for x in (cache.k_codes, cache.v_codes, cache.scales)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,Hkv,B,nodes", [(16, 1, 1, 3), (16, 8, 5, 40), (64, 3, 9, 25), (256, 2, 3, 128), (32, 8, 300, 9)])
def test_kept_paths(S, D, P, Hkv, B, nodes):
    rng = np.random.default_rng(P + D + B)
    W = pages_of(60 + nodes, P)
    cache = _cache(S, rng, B * W + 1, P, Hkv, D)
    table = rng.permutation(B * W + 1)[:B * W].reshape(B, W).astype(np.int32)
    starts = rng.integers(0, 60, B).astype(np.int32)
    counts = rng.integers(0, nodes + 1, B).astype(np.int32)
    path = np.zeros((B, nodes), np.int32)
    for b in range(B):
        path[b, :counts[b]] = np.sort(rng.choice(nodes, counts[b], replace=False))
    want = _copy(cache)
    for b in range(B):
        rows = []
        for i in range(counts[b]):
            t = starts[b] + path[b, i]
            rows.append([x[int(table[b, t // P]), :, t % P].clone() for x in (cache.k_codes, cache.v_codes, cache.scales)])
        for i, row in enumerate(rows):
            t = starts[b] + i
            for x, y in zip(want, row):
                x[int(table[b, t // P]), :, t % P] = y
    dev = lambda x: torch.from_numpy(x).cuda()   # noqa: E731
    S.kv4_keep(cache, dev(table), dev(starts), dev(path), dev(counts))
    torch.cuda.synchronize()
    for x, y in zip(_copy(cache), want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_keep_leaves_what_is_out_of_range(S):
    """Tokens outside the table, pages outside the cache, counts outside the path: nothing moves there."""
    rng = np.random.default_rng(0)
    cache = _cache(S, rng, 3, 16, 2, 64)
    before = _copy(cache)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    S.kv4_keep(cache, i32([[-1, 7], [2 ** 31 - 1, -2 ** 31]]), i32([0, 20]), i32([[1, 5], [3, 4]]), i32([2, 2]))
    S.kv4_keep(cache, i32([[0, 1]]), i32([2 ** 31 - 1]), i32([[2 ** 31 - 1]]), i32([1]))
    S.kv4_keep(cache, i32([[0, 1]]), i32([-2 ** 31]), i32([[3, 4]]), i32([9]))
    S.kv4_keep(cache, i32([[0, 1]]), i32([3]), i32([[-4]]), i32([1]))
    S.kv4_keep(cache, i32([[0, 1]]), i32([3]), i32([[5]]), i32([-3]))
    torch.cuda.synchronize()
    for x, y in zip(_copy(cache), before):
        assert torch.equal(x, y)
    S.kv4_keep(cache, i32([[0, 1]]), i32([3]), i32([[5]]), i32([100]))   # one token of the path there is
    torch.cuda.synchronize()
    assert torch.equal(cache.k_codes[0, :, 3], before[0][0, :, 8])
