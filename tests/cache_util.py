"""Helpers for the tests of the quantised cache: a small world of sequences, pages and rows, and the oracle's view of it."""
import numpy as np
import torch

from oracle import cache_ref
from paper_2605_13734_amd import kvc

DIM = 128


def rows(g, shape, dtype, spread=False):
    """Normal rows; with `spread` some channels are far larger than the others."""
    x = torch.randn(shape, generator=g, dtype=torch.float32)
    if spread:
        x = x * torch.exp(torch.randn(shape[1:], generator=g)) * torch.where(torch.rand(shape[1:], generator=g) < 0.03, 12.0, 1.0)
    return x.to(dtype)


class World:
    """Sequences with `past[s]` tokens and `new[s]` new ones; every page, table and row drawn from the seed."""

    def __init__(self, past, new, seed=0, bf16=False, kv_heads=2, per_kv=4, bits_k=4, bits_v=4, group=32, block_tokens=16, transform=0,
                 spread=True, device="cuda", limits=None):
        self.past, self.new, self.bf16, self.per_kv, self.device = past, new, bf16, per_kv, device
        self.dtype = torch.bfloat16 if bf16 else torch.float16
        self.bits_k, self.bits_v, self.group, self.rotate, self.kv_heads = bits_k, bits_v, group, bool(transform), kv_heads
        g = torch.Generator().manual_seed(seed)
        self.g = g
        n, self.total = len(past), [p + t for p, t in zip(past, new)]
        self.most_new, self.most = max(max(new), 1), max(max(self.total), 1)
        need = [(t + block_tokens - 1) // block_tokens for t in self.total]
        self.num_pages = sum(need) + 2
        order = torch.randperm(self.num_pages, generator=g)
        table = torch.full((n, max(max(need), 1)), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(need):
            table[i, :c] = order[at: at + c]
            at += c
        self.free_pages = order[at:]
        self.k = [rows(g, (t, kv_heads, DIM), self.dtype, spread) for t in self.total]
        self.v = [rows(g, (t, kv_heads, DIM), self.dtype) for t in self.total]
        self.q = rows(g, (sum(new), kv_heads * per_kv, DIM), self.dtype)
        self.table = table.to(device)
        self.new_start = self.starts(new)
        self.tokens = torch.tensor(self.total, dtype=torch.int32, device=device)
        limits = limits or {}
        self.plan = kvc.CachePlan(kvc.BF16 if bf16 else kvc.F16, kv_heads, kv_heads * per_kv, DIM, bits_k, bits_v, group, block_tokens,
                                  transform, max_batch=n, max_tokens=limits.get("tokens", self.most), max_new=self.most_new)
        self.cache = kvc.Cache(self.plan, self.num_pages, device)
        self.cache.pages.fill_(0xff)            # (what nobody wrote is NaN as a scale or zero)

    def starts(self, counts):
        return torch.tensor([0] + np.cumsum(counts).tolist(), dtype=torch.int32, device=self.device)

    def batch(self, mask=None):
        return kvc.CacheBatch(self.new_start, self.tokens, self.table, self.most_new, self.most, self.num_pages, mask)

    def past_batch(self):
        past = torch.tensor(self.past, dtype=torch.int32, device=self.device)
        return kvc.CacheBatch(self.starts(self.past), past, self.table, max(max(self.past), 1), self.most, self.num_pages)

    def all_batch(self):
        return kvc.CacheBatch(self.starts(self.total), self.tokens, self.table, self.most, self.most, self.num_pages)

    def old_rows(self):
        return [torch.cat([x[i][: self.past[i]] for i in range(len(self.past))]).to(self.device) for x in (self.k, self.v)]

    def new_rows(self):
        return [torch.cat([x[i][self.past[i]:] for i in range(len(self.past))]).to(self.device) for x in (self.k, self.v)]

    def fill(self):
        """The cache with all rows written: the past in one call, the new rows in another."""
        st = torch.cuda.current_stream().cuda_stream
        self.cache.store(self.past_batch(), *self.old_rows(), st)
        self.cache.store(self.batch(), *self.new_rows(), st)

    def held(self, s):
        """The oracle's K and V of sequence s."""
        f = lambda x: x.float().numpy()                                                        # noqa: E731
        return (cache_ref.Tensor(f(self.k[s]), self.bits_k, self.group, self.bf16, self.rotate),
                cache_ref.Tensor(f(self.v[s]), self.bits_v, self.group, self.bf16))

    def seen(self, s, mask_rows=None):
        """[new, tokens] of sequence s; mask_rows: list of Python integers, one per new row."""
        p, n = self.past[s], self.new[s]
        see = np.ones((n, p + n), dtype=bool)
        for i in range(n):
            for j in range(n):
                see[i, p + j] = j <= i if mask_rows is None else (mask_rows[i] >> j) & 1
        return see

    def mask_tensor(self, masks, words=None):
        """masks[s][i]: an integer per new row."""
        words = words or (self.most_new + 63) // 64
        out = [[(b >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for m in masks for b in m]
        return torch.tensor([[w - 2 ** 64 if w >> 63 else w for w in r] for r in out], dtype=torch.int64,
                            device=self.device).reshape(-1, words)

    def check_attention(self, out, lse, scale, masks=None):
        """Every output against the 64-bit values.  Errors: weights and values are rounded to fp16 (2^-11 each; values below 2^-14
        by 2^-25), the scores by sums of products in 32 bits (2^-19 of the largest sum of magnitudes allows for some 30 roundings),
        the output to its type."""
        at = 0
        for s in range(len(self.new)):
            n = self.new[s]
            k, v = self.held(s)
            q = self.q[at: at + n].double().numpy()
            want, want_lse, size, reach = cache_ref.attention(q, k, v, self.seen(s, None if masks is None else masks[s]), scale, self.per_kv)
            got = out[at: at + n].double().cpu().numpy()
            unit = 2.0 ** (-8 if self.bf16 else -11)
            score = reach * 2.0 ** -19
            tol = np.abs(want) * unit + size * (2.1 * 2.0 ** -11 + 2 * score[:, :, None]) + 2.0 ** -24
            bad = ~(np.abs(got - want) <= tol)
            assert not bad.any(), (s, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])
            if lse is not None:
                got_lse = lse[at: at + n].double().cpu().numpy()
                some = np.isfinite(want_lse)
                assert np.array_equal(some, np.isfinite(got_lse)) and np.all(got_lse[~some] == -np.inf)
                off = np.abs(got_lse[some] - want_lse[some])
                assert np.all(off <= score[some] + np.abs(want_lse[some]) * 2.0 ** -20 + 2.0 ** -18), off.max()
            at += n


def tree_masks(g, counts):
    """Seeded trees of drafts: (masks, accepted paths); masks[s][i] has the bits of row i's ancestors and its own."""
    masks, paths = [], []
    for n in counts:
        parent = [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)]
        m = []
        for i, p in enumerate(parent):
            m.append((1 << i) | (m[p] if p >= 0 else 0))
        node, path = n - 1, []
        while node >= 0:
            path.append(node)
            node = parent[node]
        masks.append(m)
        paths.append(path[::-1])
    return masks, paths
