"""spinq_kv4_plan where pages have been given back: entries below 0 of the page table
are no pages, so what a sequence drops of them goes on no list, in each of the plan's
forms (one CTA, a cluster, the tokens over the whole GPU).  Whole numbers: equal to
the same steps taken one sequence, one page and one token at a time."""
import numpy as np
import pytest
import torch

from test_gpu_kv4_plan import OnGpu, Server, pages_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2405_16406_gb300 import spinq
    return spinq


class Windowed(Server):
    """A Server that gives back the pages which lie before a sequence's window and behind its sinks."""

    def step(self, drop, add, total, depths=None, offset=0):
        kept = self.table.copy()
        lens = list(self.lens)
        # entries that are no pages leave no trace on the stack
        before = list(self.stack)
        P, cap = self.P, self.W * self.P
        freed = []
        for b, n in enumerate(lens):
            n = min(max(n, 0), cap)
            s = max(n - max(drop[b], 0), 0) if drop is not None else n
            freed += [int(kept[b, i]) for i in range(pages_of(s, P), pages_of(n, P)) if kept[b, i] >= 0]
        self.stack = before + freed[::-1]
        # what is left is a step that drops nothing
        self.lens = [max(min(max(n, 0), cap) - max(drop[b], 0), 0) if drop is not None else min(max(n, 0), cap)
                     for b, n in enumerate(lens)]
        return super().step(None, add, total, depths, offset)

    def give_back(self, window, sinks, which):
        for b in which:
            for i in range(max(self.lens[b] - window + 1, 0) // self.P):
                if i * self.P >= sinks and self.table[b, i] >= 0:
                    self.stack.append(int(self.table[b, i]))
                    self.table[b, i] = [-1, -(1 << 31), -7][i % 3]


class WindowedOnGpu(OnGpu):
    def take_over(self, host):
        """What the program did to the table and the list between two steps."""
        self.table.copy_(torch.from_numpy(host.table))
        self.free[:len(host.stack)] = torch.tensor(host.stack, dtype=torch.int32, device="cuda")
        self.count.fill_(len(host.stack))


def every_page_once(host):
    held = [int(p) for b, n in enumerate(host.lens) for p in host.table[b, :pages_of(n, host.P)] if p >= 0]
    assert sorted(held + host.stack) == list(range(host.capacity)), "no page lost, none twice"


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("B,longest,most,padding", [(1, 3000, 1, 0), (5, 900, 9, 3), (200, 700, 2, 0), (40, 20000, 30, 100),
                                                    (300, 2000, 3, 7), (1500, 300, 1, 0), (4096, 200, 1, 0),
                                                    (30, 6000, 500, 9000), (900, 700, 40, 50), (4096, 90, 5, 9)])
def test_windowed_sequences_grow_give_back_and_end(S, P, B, longest, most, padding):
    """Every step appends tokens, drops some, gives pages back, and now and then a sequence ends and another starts in
    its row.  (The forms: up to 1024 numbers, up to 8192 tokens, more.)"""
    rng = np.random.default_rng(B + P)
    window, sinks = int(rng.integers(1, longest)), int(rng.choice([0, 4, P, 3 * P + 1]))
    host = Windowed(rng.integers(0, longest + 1, B).tolist(), pages_of(longest + 6 * most + 1, P), P, B + 50, seed=B)
    gpu = WindowedOnGpu(S, host)
    for k in range(5):
        host.give_back(window, sinks, rng.permutation(B)[:B if k % 2 else (B + 1) // 2])
        every_page_once(host)
        gpu.take_over(host)
        ends = rng.random(B) < 0.3
        drop = np.where(ends, 1 << 20, 0).tolist()
        add = rng.integers(0, most + 1, B).tolist()
        if padding > 8192 or k == 4:   # new prompts in place of the old ones
            add = np.where(ends, rng.integers(0, longest // 4 + 2, B), add).tolist()
        # (tokens behind a page that was given back: another test)
        add = [0 if not e and n % P and host.table[b, n // P] < 0 else a for b, (a, e, n) in enumerate(zip(add, ends, host.lens))]
        total = sum(add) + padding
        want = host.step(drop, add, total)
        gpu.check(host, gpu.step(drop, add, total), want)
        every_page_once(host)
    everything = [1 << 30] * B
    gpu.check(host, gpu.step(everything, None, padding), host.step(everything, None, padding))
    assert sorted(host.stack) == list(range(host.capacity))


def test_a_window_ends_and_its_pages_serve_another(S):
    """The pages of a sequence whose first ones were given back go to the next one, which reads its own tokens."""
    window, sinks, P = 40, 4, 16
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    cache = S.kv4_pages(10, P, 1, 64)
    for x in (cache.k_codes, cache.v_codes, cache.scales):
        x.zero_()
    lens, table, free, count = i32([0, 0]), torch.full((2, 10), -1, dtype=torch.int32, device="cuda"), i32(list(range(10))), i32([10])
    g = torch.Generator(device="cuda").manual_seed(0)

    def append(add, drop=None):
        plan = S.kv4_plan(lens, i32(add), table, free, count, P, sum(add), drop=None if drop is None else i32(drop))
        k, v = (torch.randn((sum(add), 1, 64), generator=g, device="cuda").half() for _ in range(2))
        S.kv4_append(None, k, v, cache, plan.slots)
        return plan, v

    append([150, 0])
    gone = [i for i in range((150 - window + 1) // P) if i * P >= sinks]
    for i in gone:   # given back
        free[count.item()] = table[0, i]
        count += 1
        table[0, i] = -1
    plan, v = append([0, 158], [150, 0])
    torch.cuda.synchronize()
    assert plan.granted.tolist() == [1, 1] and lens.tolist() == [0, 158] and count.item() == 0
    assert sorted(table[1].tolist()) == list(range(10)) and plan.slots.min().item() >= 0
    _, read = S.kv4_read(cache, table[1:], i32([0, 158]), 158)
    step = (v.float().amax(-1) - v.float().amin(-1)) / 15
    # half a step of Eq. 1, and the output's rounding to fp16 (2^-11 of at most 8)
    assert ((v.float() - read.float()).abs().amax(-1) <= 0.51 * step + 2.0 ** -8).all()


@pytest.mark.parametrize("total", [30, 3000, 9000])
def test_no_tokens_into_a_page_that_was_given_back(S, total):
    """A sequence whose last token lies in such a page (its program dropped tokens back to before its window) is
    refused where it asks for more, as nothing could hold them; at a page's end, or without new tokens, it is not."""
    P, W = 16, 6
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    lens, drop, add = [40, 48, 33, 20, 50, 64], [3, 0, 0, 0, 17, 16], [4, 4, 0, 13, 1, 2]
    start = [37, 48, 33, 20, 33, 48]
    table = np.full((6, W), -1, np.int32)
    for b, pages in enumerate([[0, 1, -1], [2, 3, -5], [4, 5, -1], [6, 7], [8, 9, -1, 10], [11, 12, 13, -(1 << 31)]]):
        table[b, :len(pages)] = pages
    t, free, count, n = torch.from_numpy(table.copy()).cuda(), i32([20, 21, 22, 23, -1, -1, -1, -1]), i32([4]), i32(lens)
    plan = S.kv4_plan(n, i32(add), t, free, count, P, total, drop=i32(drop))
    torch.cuda.synchronize()
    granted = [0, 1, 1, 1, 0, 1]
    assert plan.granted.tolist() == granted
    assert n.tolist() == [s + a if g else s for s, a, g in zip(start, add, granted)]
    # (sequence 4 gives page 10 back, sequence 5 nothing; sequences 1, 3 and 5 take a page each)
    for b, at, page in ((1, 3, 10), (3, 2, 23), (5, 3, 22)):
        table[b, at] = page
    assert np.array_equal(t.cpu().numpy(), table)
    assert count.item() == 2 and free[:2].tolist() == [20, 21]
    want, cu = [], [0]
    for b, (s, a, g) in enumerate(zip(start, add, granted)):
        want += [int(table[b, (s + i) // P]) * P + (s + i) % P if g else -1 for i in range(a)]
        cu.append(cu[-1] + a)
    assert plan.slots.tolist() == want + [-1] * (total - len(want)) and plan.cu_tokens.tolist() == cu
