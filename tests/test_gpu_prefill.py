"""GPU tests (run with -m gpu): rotation, prompt attention, tables of pages and the quantised cache as a worker runs them together."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import cache_ref
from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, check_attention, check_rotation, heads, i32, stream

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
SCALE = DIM ** -0.5


def check_cached(out, q, k_rows, v_rows, per_kv, bits, group, rotate):
    """One new token's attention over fp16 rows that the cache holds in codes.  Tolerances as for the cache's own tests: weights and values
    rounded to fp16, scores from sums in 32 bits, the result rounded."""
    f = lambda x: x.float().cpu().numpy()                                                  # noqa: E731
    k, v = cache_ref.Tensor(f(k_rows), bits, group, False, rotate), cache_ref.Tensor(f(v_rows), bits, group, False)
    want, _, size, reach = cache_ref.attention(q[None].double().cpu().numpy(), k, v, np.ones((1, k_rows.shape[0]), dtype=bool), SCALE, per_kv)
    tol = np.abs(want) * 2.0 ** -11 + size * (2.1 * 2.0 ** -11 + 2 * reach[:, :, None] * 2.0 ** -19) + 2.0 ** -24
    off = np.abs(out[None].double().cpu().numpy() - want)
    assert np.all(off <= tol), (off / tol).max()


@pytest.mark.parametrize("lengths,steps", [((130, 1, 33), 3), ((5,), 1), ((64, 300), 2)])
def test_prefill_worker(lengths, steps):
    import prefill_worker
    (q, k, v, out, starts), done = prefill_worker.run(lengths, steps, layers=2, kv_heads=2, q_heads=6)
    for s, (a, b) in enumerate(zip(starts, starts[1:])):
        check_attention(out[a:b], None, q[a:b], k[a:b], v[a:b], SCALE, False)
        keys, values = k[a:b], v[a:b]
        for sq, sk, sv, so in done:
            keys, values = torch.cat([keys, sk[s: s + 1]]), torch.cat([values, sv[s: s + 1]])
            check_cached(so[s], sq[s], keys, values, 3, 8, 64, True)


def test_a_captured_step():
    """Tables, rotation, store and attention of single tokens, captured once and replayed as the sequences grow over pages' ends, with eager
    work in between; every replay against the same step done eagerly on a world of its own."""
    n, kv, per, lengths = 3, 2, 4, (15, 31, 60)
    frequencies = kvc.rotary_frequencies(DIM, 10000.0)

    class World:
        def __init__(self):
            self.plan = kvc.CachePlan(kvc.BF16, kv, kv * per, DIM, 4, 8, 32, 16, 0, max_batch=n, max_tokens=2000)
            self.pages = kvc.CachePages(self.plan, 40, n)
            self.cache = kvc.Cache(self.plan, 40)
            self.prompt = kvc.Prompt(kvc.PromptPlan(kvc.BF16, kv, kv * per, frequencies=frequencies, eps=1e-6, max_batch=n))
            self.start, self.tokens, self.positions = i32(*[0] * (n + 1)), i32(*[0] * n), i32(*[0] * n)
            self.one = i32(*[1] * n)
            self.q, self.k, self.v = heads(n, kv, per, True, 1)
            self.q_out, self.k_out, self.out = torch.empty_like(self.q), torch.empty_like(self.k), torch.empty_like(self.q)
            self.w = torch.ones(DIM, dtype=torch.bfloat16, device=DEVICE)
            self.batch = kvc.CacheBatch(self.start, self.tokens, self.pages.table, 1, 2000, 40)
            rows = i32(*[0] * sum(lengths))
            self.pages.advance(self.start, self.tokens, fresh=i32(*lengths), max_new=60, positions=rows, stream=stream())
            q, k, v = heads(sum(lengths), kv, per, True, 2)
            self.prompt.rotate(None, k, rows, k_weight=self.w, stream=stream())
            self.cache.store(kvc.CacheBatch(self.start, self.tokens, self.pages.table, 60, 2000, 40), k, v, stream())

        def step(self):
            self.pages.advance(self.start, self.tokens, fresh=self.one, max_new=1, positions=self.positions, stream=stream())
            self.prompt.rotate(self.q, self.k, self.positions, self.q_out, self.k_out, self.w, self.w, stream=stream())
            self.cache.store(self.batch, self.k_out, self.v, stream())
            self.cache.attend(self.batch, self.q_out, self.out, SCALE, stream=stream())

        def state(self):
            return [self.out, self.q_out, self.tokens, self.pages.held, self.pages.free, self.pages.table, self.cache.pages]

    captured, eager = World(), World()
    for w in (captured, eager):
        w.step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        captured.step()
    for i in range(9):
        for w in (captured, eager):
            for x, y in zip((w.q, w.k, w.v), heads(n, kv, per, True, 100 + i)):
                x.copy_(y)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for x, y in zip(captured.state(), eager.state()):
            assert torch.equal(x, y), i
        assert eager.positions.tolist() == [t + 1 + i for t in lengths] == captured.positions.tolist()
    for w in (captured, eager):
        assert not any(s.any() for s in (w.cache.status, w.pages.status, w.prompt.status))


def test_rows_behind_the_last_sequence():
    """A padded batch: rows that belong to nobody have position -1 and go through all calls untouched."""
    kv, per, rows = 2, 2, 90
    plan = kvc.CachePlan(kvc.F16, kv, kv * per, DIM, 8, 8, 64, 16, max_batch=3, max_tokens=200)
    pages, cache = kvc.CachePages(plan, 20, 3), kvc.Cache(plan, 20)
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, kv, kv * per, max_batch=3))
    start, tokens, positions = i32(0, 0, 0, 0), i32(0, 0, 0), i32(*[5] * rows)
    slots = torch.zeros(rows, dtype=torch.int64, device=DEVICE)
    pages.advance(start, tokens, fresh=i32(33, 300, 20), max_new=300, rows=rows, positions=positions, slots=slots, stream=stream())
    # (the second is longer than the plan allows: it is left out, with its rows and with those that follow and do not fit)
    assert pages.status.tolist() == [0, kvc.DEV_BAD_ROW, kvc.DEV_BAD_ROW] and tokens.tolist() == [33, -1, -1]
    assert positions.tolist() == list(range(33)) + [-1] * 57 and slots.tolist() == list(range(16)) + list(range(16, 33)) + [-1] * 57
    q, k, v = heads(rows, kv, per, False, 4)
    q0, k0 = q.clone(), k.clone()
    prompt.rotate(q, k, positions, stream=stream())
    assert torch.equal(q[33:], q0[33:]) and torch.equal(k[33:], k0[33:])
    check_rotation(q[:33], q0[:33], None, np.arange(33), kvc.rotary_frequencies(DIM), False, 1.0, None, False)
    out = torch.full_like(q, 77.0)
    prompt.attend(kvc.PromptBatch(start, 33), q, k, v, out, SCALE, stream=stream())
    assert prompt.status.tolist() == [0, kvc.DEV_BAD_ROW, kvc.DEV_BAD_ROW] and (out[33:] == 77).all()
    check_attention(out[:33], None, q[:33], k[:33], v[:33], SCALE, False)
    cache.store(kvc.CacheBatch(start, tokens, pages.table, 300, 200, 20), k, v, stream())
    assert cache.status.tolist() == [0, kvc.DEV_BAD_ROW, kvc.DEV_BAD_ROW]
    back = torch.full_like(k, 77.0), torch.full_like(v, 77.0)
    cache.load(kvc.CacheBatch(i32(0, 33), i32(33), pages.table[:1], 33, 200, 20), *back, stream())
    assert ((back[1][:33].float() - v[:33].float()).abs() <= 0.04).all() and (back[1][33:] == 77).all()
