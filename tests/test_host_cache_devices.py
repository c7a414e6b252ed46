"""CPU-only checks of where the tensors of the quantised cache's calls may lie.  No kernel is launched here."""
import os

import pytest
import torch

from paper_2605_13734_amd import kvc


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvc.LIB_PATH):
        from paper_2605_13734_amd import build
        build.build()
    return kvc.load()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def world():
    """A cache whose tensors, like all others here, are in host memory, and well-formed arguments of its four calls."""
    plan = kvc.CachePlan(dtype=kvc.F16, kv_heads=2, q_heads=8, max_tokens=1000, max_new=4, max_batch=3)
    cache = kvc.Cache(plan, 10, "cpu")
    batch = kvc.CacheBatch(i32(0, 2), i32(42), torch.zeros(1, 3, dtype=torch.int32), 2, 42, 10)
    return cache, batch, torch.zeros(2, 2, 128, dtype=torch.float16), torch.zeros(2, 8, 128, dtype=torch.float16)


def test_a_cache_in_host_memory_refuses_its_calls(lib):
    """All tensors are on one device, which is no GPU: nothing is handed to a kernel."""
    cache, batch, rows, q = world()
    for call in (lambda: cache.store(batch, rows, rows.clone()), lambda: cache.load(batch, rows, rows.clone()),
                 lambda: cache.keep(batch, i32(0, 1), i32(0)), lambda: cache.attend(batch, q, q.clone(), 0.1),
                 lambda: cache.attend(batch, q, q.clone(), 0.1, torch.zeros(2, 8))):
        with pytest.raises(ValueError):
            call()
    assert not cache.status.any()
