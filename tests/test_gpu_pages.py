"""GPU tests (run with -m gpu): the sequences of a step - lengths, starts, positions, slots, pages taken and given back - against a
definition in plain Python."""
import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, Pages, i32, stream

pytestmark = pytest.mark.gpu


class Both:
    """The GPU's tables and the definition's, through the same steps."""

    def __init__(self, n, num_pages, block_tokens, max_tokens, seed=0):
        self.n, self.g = n, np.random.default_rng(seed)
        self.plan = kvc.CachePlan(kvc.F16, 1, 1, block_tokens=block_tokens, max_tokens=max_tokens, max_batch=n)
        self.gpu = kvc.CachePages(self.plan, num_pages, n)
        free = self.g.permutation(num_pages).tolist()
        self.gpu.set_free(torch.tensor(free, dtype=torch.int32))
        self.want = Pages(n, num_pages, block_tokens, max_tokens, free)
        self.table = np.full(self.gpu.table.shape, -1)
        self.start, self.tokens = i32(*[0] * (n + 1)), i32(*[0] * n)

    def step(self, kept, fresh, max_new, rows, arrays=True, max_tokens=None):
        words = lambda x: None if x is None else i32(*x)                                    # noqa: E731
        positions = torch.full((rows,), -7, dtype=torch.int32, device=DEVICE) if arrays else None
        slots = torch.full((rows,), -7, dtype=torch.int64, device=DEVICE) if arrays else None
        self.gpu.status.zero_()
        self.gpu.advance(self.start, self.tokens, words(kept), words(fresh), max_new, max_tokens, positions, slots, rows, stream())
        start, tokens, at, slot, status = self.want.advance(kept, fresh, max_new, rows, max_tokens)
        assert self.start.tolist() == start and self.tokens.tolist() == tokens
        assert self.gpu.status.tolist() == status
        if arrays:
            assert positions.tolist() == at and slots.tolist() == slot
        self.compare()
        return status

    def compare(self):
        w = self.want
        for s, p in enumerate(w.pages):
            self.table[s, : len(p)] = p      # (places behind a sequence's pages stay as they were)
        assert np.array_equal(self.gpu.table.cpu().numpy(), self.table)
        assert self.gpu.held.tolist() == w.held
        assert self.gpu.free[:4].tolist() == [len(w.stack), 0, 0, 0]
        assert self.gpu.free_pages[: len(w.stack)].tolist() == w.stack


@pytest.mark.parametrize("n,num_pages,block_tokens,max_tokens,most", [(1, 9, 16, 140, 40), (3, 30, 16, 200, 70), (40, 200, 32, 300, 90), (65, 700, 64, 4000, 1500),
                                                                      (1025, 9000, 16, 300, 40), (4096, 20000, 16, 99, 12)])
def test_random_steps(n, num_pages, block_tokens, max_tokens, most):
    """Prompts, drafts kept in part, sequences that end, too few pages now and then."""
    b = Both(n, num_pages, block_tokens, max_tokens, seed=n)
    seen = set()
    for step in range(12 if n < 1000 else 5):
        held = np.array(b.want.held)
        ends = b.g.random(n) < 0.3
        kept = np.where(ends, 0, held - np.minimum(held, b.g.integers(0, 20, n) * (b.g.random(n) < 0.5)))
        fresh = np.minimum(np.where(b.g.random(n) < 0.2, b.g.integers(0, most + 1, n), b.g.integers(0, 3, n)), max_tokens - kept)
        total = int(fresh.sum())
        kept, fresh = kept.tolist(), fresh.tolist()
        if step % 4 == 3:
            kept = None
            fresh = np.minimum(b.g.integers(0, 3, n), max_tokens - held).tolist()
            total = sum(fresh)
        seen |= set(b.step(kept, fresh, most, total + int(b.g.integers(0, 50)), arrays=step != 5))
    assert kvc.DEV_BAD_ROW not in seen
    b.step([0] * n, None, 0, 0, arrays=False)
    assert b.gpu.free[0] == num_pages and sorted(b.gpu.free_pages.tolist()) == list(range(num_pages))


def test_there_and_back():
    """Pages taken and given back leave the stack as it was, whichever side has more of them."""
    b = Both(6, 60, 16, 300, seed=3)
    b.step(None, [100, 0, 47, 16, 1, 0], 200, 164)
    held, stack, table = list(b.want.held), list(b.want.stack), b.gpu.table.clone()
    for fresh, kept in (([33, 20, 1, 0, 15, 100], None), ([0, 150, 0, 0, 3, 20], [0, 0, 0, 16, 1, 0]), ([0, 5, 0, 1, 0, 0], [0, 0, 47, 0, 0, 0])):
        b.step(kept, fresh, 200, sum(fresh))
        keep = [min(h, k) for h, k in zip(held, kept or held)]
        b.step(keep, [h - k for h, k in zip(held, keep)], 200, 300)
        assert b.want.stack == stack and b.want.held == held and b.gpu.free_pages[: len(stack)].tolist() == stack
    same = torch.tensor([[i < (h + 15) // 16 for i in range(b.gpu.table.shape[1])] for h in held], device=DEVICE)
    assert torch.equal(b.gpu.table[same], table[same])


def test_numbers_that_do_not_fit():
    """Left out and reported, with what they hold; the others go on.  The new rows of one that is left out still count."""
    b = Both(9, 50, 16, 200, seed=4)
    b.step(None, [40, 20, 30, 10, 50, 60, 16, 0, 5], 100, 231)
    top = 2 ** 31 - 1
    status = b.step([41, -1, 30, 10, 50, 0, 16, 0, 5], [1, 1, -3, 101, 150, 30, 1, 1, top], 100, 300)
    bad = kvc.DEV_BAD_ROW
    assert status == [bad, bad, bad, bad, bad, 0, 0, 0, bad]
    assert b.step(None, [1] * 9, 100, 4) == [0] * 4 + [bad] * 5            # room for four rows
    assert b.step(None, [1] * 9, 0, 9) == [bad] * 9
    assert b.step(None, [1] * 9, 5, 9, max_tokens=30) == [bad if h > 29 else 0 for h in (41, 21, 31, 11, 50, 30, 17, 1, 5)]
    b.step(None, [100] * 9, 100, 900)


def test_too_few_pages():
    """Those before get theirs, those that need none go on, and what others give back counts."""
    b = Both(5, 10, 16, 200, seed=5)
    none = kvc.DEV_NO_PAGE
    assert b.step(None, [70, 60, 20, 0, 0], 100, 150) == [0, 0, none, 0, 0]            # 5 + 4 pages; one is left
    assert b.step(None, [10, 5, 0, 17, 16], 100, 48) == [0, 0, 0, none, none]          # 0, 1 (65 tokens: a fifth), 0, 2, 1 wanted
    assert b.step([80, 0, 0, 0, 0], [0, 20, 0, 17, 16], 100, 53) == [0, 0, 0, 0, 0]
    assert b.step([0, 0, 0, 0, 0], [160, 0, 0, 0, 1], 160, 161) == [none, 0, 0, 0, 0]  # the fifth keeps a page
    assert b.step([0, 0, 0, 0, 0], [160, 0, 0, 0, 0], 160, 160) == [0, 0, 0, 0, 0]


def test_pages_that_are_no_pages():
    """Numbers outside the pool in the stack and in a table: passed on as -1 and reported, nothing outside is touched."""
    plan = kvc.CachePlan(kvc.F16, 1, 1, block_tokens=16, max_tokens=100, max_batch=3)
    p = kvc.CachePages(plan, 8, 3)
    p.set_free(torch.tensor([1, 99, 2, -5], dtype=torch.int32))
    start, tokens = i32(0, 0, 0, 0), i32(0, 0, 0)
    positions, slots = i32(*[0] * 52), torch.zeros(52, dtype=torch.int64, device=DEVICE)
    p.advance(start, tokens, None, i32(17, 3, 32), 40, None, positions, slots, stream=stream())
    assert p.status.tolist() == [kvc.DEV_BAD_BLOCK, kvc.DEV_BAD_BLOCK, kvc.DEV_NO_PAGE]
    assert p.table[:, :2].tolist() == [[-1, 2], [-1, -1]] + [[-1, -1]] and tokens.tolist() == [17, 3, -1]
    assert slots.tolist() == [-1] * 16 + [32] + [-1] * 35 and positions.tolist() == list(range(17)) + [0, 1, 2] + [-1] * 32
    assert p.free[:4].tolist() == [1, 0, 0, 0] and p.free[4] == 1
    p.status.zero_()
    p.advance(start, tokens, i32(0, 0, 0), None, 0, rows=0, stream=stream())
    assert p.status.tolist() == [kvc.DEV_BAD_BLOCK, kvc.DEV_BAD_BLOCK, 0]
    assert p.free[:8].tolist() == [4, 0, 0, 0, 1, -1, 2, -1]


def test_a_count_outside_the_pool():
    """A number of free pages beyond the pool's, or more given back than there is room: nothing is written behind the stack."""
    plan = kvc.CachePlan(kvc.F16, 1, 1, block_tokens=16, max_tokens=100, max_batch=2)
    p = kvc.CachePages(plan, 4, 2)
    p.free = torch.cat([p.free, i32(77, 77)])
    p._free = p.free.data_ptr()
    p.free[0] = 1000
    start, tokens = i32(0, 0, 0), i32(0, 0)
    p.advance(start, tokens, None, i32(33, 30), 40, stream=stream())
    assert p.status.tolist() == [0, kvc.DEV_NO_PAGE] and p.free[0] == 1 and p.table[0, :3].tolist() == [0, 1, 2]
    p.free[0] = 3
    p.advance(start, tokens, i32(0, 0), None, 0, stream=stream())
    assert p.free[0] == 4 and p.free[-2:].tolist() == [77, 77]
    p.free[0] = -9
    p.advance(start, tokens, None, i32(1, 0), 40, stream=stream())
    assert p.status.tolist() == [kvc.DEV_NO_PAGE, kvc.DEV_NO_PAGE] and p.free[0] == 0


def test_the_largest_numbers():
    """Sums of new tokens beyond 32 bits: the rows that there is room for are right."""
    plan = kvc.CachePlan(kvc.F16, 1, 1, block_tokens=4096, max_tokens=0x7fffff00, max_batch=5)
    p = kvc.CachePages(plan, 600000, 5)
    start, tokens = i32(*[0] * 6), i32(*[0] * 5)
    positions = i32(*[0] * 20)
    big = 0x7fffff00
    p.advance(start, tokens, None, i32(5, big, 3, big, big), 0x7fffffff, None, positions, stream=stream())
    assert start.tolist() == [0, 5, 5 + big, 8 + big, 2 ** 31 - 1, 2 ** 31 - 1]
    assert tokens.tolist() == [5, -1, -1, -1, -1] and p.status.tolist() == [0] + [kvc.DEV_BAD_ROW] * 4
    assert positions.tolist() == [0, 1, 2, 3, 4] + [-1] * 15
    p.status.zero_()
    p.advance(start, tokens, None, i32(0, big, 0, 0, 0), 0x7fffffff, stream=stream())
    assert tokens.tolist() == [5, big, 0, 0, 0] and not p.status.any()
    assert p.free[0] == 600000 - 1 - 0x7fffff00 // 4096 - 1 and p.table[1, 0x7fffff00 // 4096] == 0x7fffff00 // 4096 + 1


def test_captured_and_replayed():
    """A step of one new token, replayed as the sequences grow, with eager steps in between."""
    b = Both(7, 80, 16, 150, seed=6)
    b.step(None, [5, 15, 16, 17, 31, 32, 0], 40, 116)
    one, positions = i32(*[1] * 7), i32(*[0] * 7)
    slots = torch.zeros(7, dtype=torch.int64, device=DEVICE)
    call = lambda: b.gpu.advance(b.start, b.tokens, None, one, 1, None, positions, slots, stream=stream())      # noqa: E731
    call()
    b.want.advance(None, [1] * 7, 1, 7)
    b.compare()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(40):
        graph.replay()
        start, tokens, at, slot, _ = b.want.advance(None, [1] * 7, 1, 7)
        assert positions.tolist() == at and slots.tolist() == slot and b.tokens.tolist() == tokens
        b.compare()
        if i % 13 == 5:
            b.step([max(h - 9, 0) for h in b.want.held], [3] * 7, 3, 25)


def test_large_prompts():
    """Rows and pages that many workgroups share."""
    b = Both(5, 20000, 16, 70000, seed=7)
    b.step(None, [70000, 1, 0, 65537, 4096], 70000, 139700)
    b.step([0, 1, 0, 30000, 4096], [0, 69999, 5, 40000, 0], 70000, 110004)
