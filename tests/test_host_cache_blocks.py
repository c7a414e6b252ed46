"""CPU-only checks of the size of the blocks of query rows that an attention over the quantised cache takes.  No kernel is launched here."""
import os

import pytest

from paper_2605_13734_amd import kvc


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvc.LIB_PATH):
        from paper_2605_13734_amd import build
        build.build()
    return kvc.load()


def plan(kv_heads, per_kv, **kw):
    return kvc.CachePlan(**{**dict(dtype=kvc.F16, kv_heads=kv_heads, q_heads=kv_heads * per_kv, max_tokens=1 << 22, max_new=4096, max_batch=64), **kw})


def test_calls_without_blocks(lib):
    p = plan(2, 4)
    assert lib.kvc_cache_block_rows(None, 1, 1, 1) == 0
    for n, new, tokens in [(0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1), (65, 1, 1), (1, 4097, 8192), (1, 1, (1 << 22) + 1)]:
        assert p.block_rows(n, new, tokens) == 0
    assert p.block_rows(1, 4096, 1) == 16                      # (new rows are tokens)


@pytest.mark.parametrize("n,rows,tokens,want", [(1, 128, 2000, 16), (1, 128, 16000, 32), (1, 512, 2000, 16), (4, 256, 1000, 32), (4, 256, 8000, 32),
                                                (4, 256, 16000, 128), (8, 512, 500, 128), (8, 512, 4000, 128)])
def test_the_size_that_was_the_fastest(lib, n, rows, tokens, want):
    """Eight KV heads, four query heads each: measured calls."""
    assert plan(8, 4).block_rows(n, rows // 4, tokens + rows // 4) == want


def test_rows_that_larger_blocks_would_not_fill(lib):
    for kv_heads, per_kv in ((1, 1), (8, 4), (2, 16)):
        p = plan(kv_heads, per_kv)
        for n in (1, 7, 64):
            for tokens in (100, 5000, 1 << 22):
                for new in range(1, 65):
                    got, rows = p.block_rows(n, new, tokens), new * per_kv
                    assert got == 16 if rows <= 16 else got in (16, 32) if rows <= 64 else got in (16, 32, 128)


def test_loose_bounds_take_larger_blocks(lib):
    p = plan(8, 4)
    assert p.block_rows(1, 32, 2048) == 16 and p.block_rows(1, 32, 1 << 17) == 128
