"""CPU-only checks of the quantised cache: plans, sizes and the arguments that its calls refuse before anything is launched, and the
oracle's quantiser against plain facts.  No kernel is launched here."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import cache_ref
from paper_2605_13734_amd import kvc


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvc.LIB_PATH):
        from paper_2605_13734_amd import build
        build.build()
    return kvc.load()


def plan(**kw):
    return kvc.CachePlan(**{**dict(dtype=1, kv_heads=2, q_heads=8, max_tokens=1000, max_new=4, max_batch=3), **kw})


def test_plans(lib):
    for kw in [dict(), dict(bits_k=8, bits_v=8, group=128, block_tokens=4096, transform=1, dtype=2), dict(q_heads=2), dict(max_tokens=0)]:
        plan(**kw)
    for kw in [dict(dtype=3), dict(group=16), dict(group=96), dict(kv_heads=0), dict(q_heads=7), dict(q_heads=0), dict(max_new=0),
               dict(max_batch=0), dict(max_tokens=-1), dict(block_tokens=0)]:
        with pytest.raises(kvc.KvcError) as e:
            plan(**kw)
        assert e.value.status == -1, kw
    for kw in [dict(bits_k=2), dict(bits_v=16), dict(head_dim=64), dict(block_tokens=8), dict(block_tokens=48), dict(block_tokens=8192),
               dict(transform=2), dict(max_batch=65536)]:
        with pytest.raises(kvc.KvcError) as e:
            plan(**kw)
        assert e.value.status == -2, kw
    for kw in [dict(max_tokens=1 << 31), dict(max_new=1 << 28), dict(kv_heads=64, q_heads=64, max_new=1 << 25)]:
        with pytest.raises(kvc.KvcError) as e:
            plan(**kw)
        assert e.value.status == -3, kw


def test_null_plans(lib):
    out = C.c_void_p(7)
    assert lib.kvc_cache_plan(None, 1, 1, 1, C.byref(out)) == -1 and not out.value
    assert lib.kvc_cache_plan(C.byref(kvc.CacheConfig(1, 4, 4, 0, 32, 16, 1, 1, 128)), 1, 1, 1, None) == -1
    assert lib.kvc_cache_page_bytes(None) == 0 and lib.kvc_cache_workspace_size(None) == 0
    lib.kvc_cache_plan_free(None)


@pytest.mark.parametrize("bits_k,bits_v,group,block_tokens,heads", [(4, 4, 32, 16, 8), (8, 4, 64, 64, 3), (4, 8, 128, 32, 1), (8, 8, 32, 256, 4)])
def test_page_bytes(lib, bits_k, bits_v, group, block_tokens, heads):
    """Codes and, per token and group, four fp16 numbers: nothing else."""
    p = plan(bits_k=bits_k, bits_v=bits_v, group=group, block_tokens=block_tokens, kv_heads=heads, q_heads=heads)
    assert p.page_bytes() == heads * block_tokens * (16 * (bits_k + bits_v) + 128 // group * 8)


def test_workspace(lib):
    assert plan(max_tokens=64).workspace_size() == 0
    small, long, wide = plan(max_tokens=5000), plan(max_tokens=1 << 20), plan(max_tokens=1 << 20, max_batch=4096, max_new=64)
    assert 0 < small.workspace_size() <= long.workspace_size() <= wide.workspace_size() < 64 << 20


@pytest.mark.parametrize("kv_heads,per_kv,max_new", [(8, 8, 64), (3, 5, 40), (1, 1, 300), (40, 2, 9), (128, 1, 1), (7, 16, 100)])
def test_workspace_is_enough_for_every_call_of_a_plan(lib, kv_heads, per_kv, max_new):
    """Calls with fewer sequences or new tokens than the plan has are accepted (they end at the device that is not there)."""
    if torch.cuda.is_available():
        pytest.skip("would launch")
    p = plan(kv_heads=kv_heads, q_heads=kv_heads * per_kv, max_new=max_new, max_tokens=1 << 20, max_batch=300)
    for n in (1, 2, 31, 256, 257, 300):
        for new in sorted(set(range(1, max_new + 1, 7)) | {1, 2, 3, 4, 5, 8, 16, 17, max_new}):
            if new > max_new:
                continue
            a = Args(p)
            a.batch.n, a.batch.max_new, a.batch.max_tokens, a.batch.table_stride = n, new, 1 << 20, 1 << 16
            assert a.calls(lib)["attend"]() == -6, (n, new)


class Args:
    """Arguments of a call that is well formed but for what a test changes (addresses are never followed)."""

    def __init__(self, p):
        self.p = p
        self.batch = kvc.CacheSequences(2, 4, 1000, 0x1000, 0x2000, 0x3000, 63, None, 0, 200)
        self.rows = kvc.CacheRows(0x10000, 0x20000, 8, 256, 128)
        self.queries = kvc.CacheQueries(0x10000, 0x20000, None, 8, 1024, 128, 1024, 128, 0.1)
        self.pages, self.status, self.workspace = 0x40000, 0x5000, 0x60000
        self.keep_start, self.keep, self.keep_rows = 0x7000, 0x8000, 4

    def calls(self, lib):
        b = C.byref(self.batch)
        return {"store": lambda: lib.kvc_cache_store(self.p._h, b, C.byref(self.rows), self.pages, self.status, None),
                "load": lambda: lib.kvc_cache_load(self.p._h, b, C.byref(self.rows), self.pages, self.status, None),
                "keep": lambda: lib.kvc_cache_keep(self.p._h, b, self.keep_start, self.keep, self.keep_rows, self.pages, self.status, None),
                "attend": lambda: lib.kvc_cache_attend(self.p._h, b, C.byref(self.queries), self.pages, self.status, self.workspace, None)}


BATCH = [(dict(n=-1), -1), (dict(n=4), -3), (dict(max_new=-1), -1), (dict(max_tokens=1001), -3), (dict(max_tokens=-1), -1),
         (dict(new_start=None), -1), (dict(tokens=None), -1), (dict(block_table=None), -1), (dict(new_start=0x1002), -1),
         (dict(table_stride=62), -1), (dict(table_stride=-1), -1), (dict(num_pages=-1), -1), (dict(mask=0x9000, mask_words=0), -1),
         (dict(mask=0x9004, mask_words=1), -1)]


@pytest.mark.parametrize("change,want", BATCH, ids=[str(c) for c, _ in BATCH])
def test_sequences_that_are_refused(lib, change, want):
    for name in ("store", "load", "keep", "attend"):
        a = Args(plan())
        for k, v in change.items():
            setattr(a.batch, k, v)
        assert a.calls(lib)[name]() == want, name


def test_new_tokens_of_an_attention(lib):
    """The plan bounds them for the attention alone."""
    a = Args(plan())
    a.batch.max_new = 5
    assert a.calls(lib)["attend"]() == -3


def test_tensors_that_are_refused(lib):
    for name, part, change in [(n, "rows", c) for n in ("store", "load") for c in (dict(k=None), dict(v=None), dict(k=0x10008), dict(v=0x20002),
                                                                                   dict(rows=-1), dict(stride_row=130), dict(stride_head=4))] + \
                              [("attend", "queries", c) for c in (dict(q=None), dict(out=None), dict(q=0x10008), dict(out=0x20004), dict(lse=0x9002),
                                                                  dict(rows=-1), dict(q_stride_row=1025), dict(q_stride_head=4),
                                                                  dict(out_stride_row=1028), dict(out_stride_head=100), dict(scale=float("nan")),
                                                                  dict(scale=float("inf")))]:
        a = Args(plan())
        for k, v in change.items():
            setattr(getattr(a, part), k, v)
        assert a.calls(lib)[name]() == -1, (name, change)
    for change in (dict(pages=None), dict(pages=0x40008), dict(status=None), dict(status=0x5002)):
        for name in ("store", "load", "keep", "attend"):
            a = Args(plan())
            for k, v in change.items():
                setattr(a, k, v)
            assert a.calls(lib)[name]() == -1, (name, change)
    for change in (dict(keep_start=None), dict(keep=None), dict(keep_rows=-1), dict(keep=0x8002), dict(keep_rows=1 << 31)):
        a = Args(plan())
        for k, v in change.items():
            setattr(a, k, v)
        assert a.calls(lib)["keep"]() == -1, change
    a = Args(plan())
    assert a.p.workspace_size() > 0
    for w in (None, 0x60004):
        a.workspace = w
        assert a.calls(lib)["attend"]() == -1
    a = Args(plan())
    b = C.byref(a.batch)
    assert lib.kvc_cache_store(None, b, C.byref(a.rows), a.pages, a.status, None) == -1
    assert lib.kvc_cache_store(a.p._h, None, C.byref(a.rows), a.pages, a.status, None) == -1
    assert lib.kvc_cache_load(a.p._h, b, None, a.pages, a.status, None) == -1
    assert lib.kvc_cache_attend(a.p._h, b, None, a.pages, a.status, a.workspace, None) == -1


def test_calls_with_nothing_to_do(lib):
    for change in (dict(n=0), dict(max_new=0), dict(max_tokens=0)):
        a = Args(plan())
        for k, v in change.items():
            setattr(a.batch, k, v)
        a.batch.new_start = a.batch.tokens = None
        for name, call in a.calls(lib).items():
            assert call() == 0, (name, change)


def test_binding_refuses_what_the_library_cannot_see(lib):
    p = plan()
    cache = kvc.Cache(p, 10, "cpu")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)                        # noqa: E731
    table = torch.zeros(2, 63, dtype=torch.int32)
    with pytest.raises(TypeError):
        kvc.CacheBatch(i32(0, 1, 2).long(), i32(5, 5), table, 1, 10, 10)
    with pytest.raises(ValueError):
        kvc.CacheBatch(i32(0, 1), i32(5, 5), table, 1, 10, 10)
    with pytest.raises(ValueError):
        kvc.CacheBatch(i32(0, 1, 2), i32(5, 5), table.t(), 1, 10, 10)
    with pytest.raises(ValueError):
        kvc.CacheBatch(i32(0, 1, 2), i32(5, 5), table, 1, 10, 10, torch.zeros(2, 1, dtype=torch.int32))
    b = kvc.CacheBatch(i32(0, 1, 2), i32(5, 5), table, 1, 10, 10, torch.zeros(2, 1, dtype=torch.int64))
    row = lambda n, h, d=128, t=torch.float16: torch.zeros(n, h, d, dtype=t)   # noqa: E731
    for k, v in [(row(2, 3), row(2, 3)), (row(2, 2, 64), row(2, 2, 64)), (row(2, 2, t=torch.bfloat16), row(2, 2, t=torch.bfloat16)),
                 (row(2, 2), row(3, 2)), (row(2, 2), row(2, 4)[:, ::2]), (row(128, 2, 2).transpose(0, 2), row(128, 2, 2).transpose(0, 2))]:
        with pytest.raises(ValueError):
            cache.store(b, k, v)
        with pytest.raises(ValueError):
            cache.load(b, k, v)
    for q, out, lse in [(row(2, 2), row(2, 8), None), (row(2, 8), row(3, 8), None), (row(3, 8), row(3, 8), None),
                        (row(2, 8), row(2, 8), torch.zeros(2, 8, dtype=torch.float16)), (row(2, 8), row(2, 8), torch.zeros(8, 2))]:
        with pytest.raises(ValueError):
            cache.attend(b, q, out, 1.0, lse)
    for start, keep in [(i32(0, 1), i32(0)), (i32(0, 1, 1).long(), i32(0)), (i32(0, 1, 1), i32(0).float())]:
        with pytest.raises(ValueError):
            cache.keep(b, start, keep)
    with pytest.raises(ValueError):
        cache.store(kvc.CacheBatch(i32(0, 1, 2), i32(5, 5), table, 1, 10, 11), row(2, 2), row(2, 2))
    with pytest.raises(ValueError):
        kvc.Cache(p, 10, "cpu", workspace=torch.zeros(64, dtype=torch.uint8))


def test_oracle_quantiser():
    """Codes reach both ends of their range, errors are half a step (and what the 16-bit zero and scale add), the rotation is its own
    inverse up to the quantiser's error."""
    g = np.random.default_rng(0)
    x = g.standard_normal((50, 128)).astype(np.float16).astype(np.float32)
    for bits, group in ((4, 32), (8, 128)):
        t = cache_ref.Tensor(x, bits, group, False)
        assert t.code.min() == 0 and t.code.max() == 2 ** bits - 1
        assert np.all(np.abs(t.values() - x) <= t.scale * (0.5 + 2.0 ** (bits - 11)) + 2.0 ** -12)
        r = cache_ref.Tensor(x, bits, group, False, rotate=True)
        back = r.read_back(False)
        assert np.sqrt(np.mean((back - x) ** 2)) < 1.2 * np.sqrt(np.mean(r.scale ** 2) * 128 / 12) / 11.3 * 2 ** 0.5 * 1.2
    h = cache_ref.hadamard()
    assert np.allclose(cache_ref.transform32(x, 0.125), x @ h / 8, atol=1e-4)


def test_oracle_attention():
    """Two equal keys share the weight; a token that is not seen has none; one that sees nothing gives zeros."""
    k = cache_ref.Tensor(np.ones((3, 1, 128), np.float32), 8, 32, False)
    v = cache_ref.Tensor(np.stack([np.full((1, 128), f, np.float32) for f in (1, 3, 100)]), 8, 32, False)
    seen = np.array([[True, True, False], [False, False, False]])
    out, lse, _, _ = cache_ref.attention(np.ones((2, 1, 128)), k, v, seen, 0.01, 1)
    assert np.allclose(out[0], 2.0) and np.all(out[1] == 0) and lse[1, 0] == -np.inf
    assert np.isclose(lse[0, 0], 1.28 + np.log(2))


def test_calls_too_large_for_a_launch(lib):
    """What no launch can hold is refused before anything starts: 2^31 new rows of 64 heads, 5000 blocks of rows for 40 heads and more
    sequences than are divided."""
    p = plan(kv_heads=64, q_heads=64, max_tokens=0x7fffff00, max_new=1)
    a = Args(p)
    a.batch.max_new, a.batch.max_tokens, a.batch.table_stride = 0x7fffffff, 0x7fffff00, 1 << 27
    assert a.calls(lib)["store"]() == -3 and a.calls(lib)["load"]() == -3
    p = plan(kv_heads=40, q_heads=40, max_tokens=640000, max_new=640000, max_batch=300)
    a = Args(p)
    a.batch.n, a.batch.max_new, a.batch.max_tokens, a.batch.table_stride = 300, 640000, 640000, 40000
    assert a.calls(lib)["attend"]() == -3
