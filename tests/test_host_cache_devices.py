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


class OnSecondDevice(torch.Tensor):
    """A tensor that says that it is on the second of two devices."""
    is_cuda = True

    def get_device(self):
        return 1


class Recorder:
    """The library, but for the four calls, which note the current device."""

    def __init__(self, lib, at):
        self.lib, self.at, self.seen = lib, at, []

    def __getattr__(self, name):
        if name not in ("kvc_cache_store", "kvc_cache_load", "kvc_cache_keep", "kvc_cache_attend"):
            return getattr(self.lib, name)

        def call(*args):
            self.seen.append((name, self.at[-1]))
            return 0
        return call


def test_the_calls_of_a_cache_go_to_its_device(lib, monkeypatch):
    """Two devices, the first of which is current: a call makes the cache's the current one while it launches."""
    at = [0]

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            at.append(self.device)

        def __exit__(self, *_):
            at.pop()

    zeros = torch.zeros
    second = lambda *a, device=None, **kw: zeros(*a, **kw).as_subclass(OnSecondDevice)       # noqa: E731
    recorder = Recorder(lib, at)
    monkeypatch.setattr(torch, "zeros", second)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    plan = kvc.CachePlan(dtype=kvc.F16, kv_heads=2, q_heads=8, max_tokens=1000, max_new=4, max_batch=3)
    monkeypatch.setattr(kvc, "_lib", recorder)
    cache = kvc.Cache(plan, 10, "cuda:1")
    words = lambda *v: i32(*v).as_subclass(OnSecondDevice)                                   # noqa: E731
    batch = kvc.CacheBatch(words(0, 2), words(42), second(1, 3, dtype=torch.int32), 2, 42, 10)
    rows, q = second(2, 2, 128, dtype=torch.float16), second(2, 8, 128, dtype=torch.float16)
    cache.store(batch, rows, rows)
    cache.load(batch, rows, rows)
    cache.keep(batch, words(0, 1), words(0))
    cache.attend(batch, q, q, 0.1)
    assert recorder.seen == [("kvc_cache_store", 1), ("kvc_cache_load", 1), ("kvc_cache_keep", 1), ("kvc_cache_attend", 1)]
    assert at == [0]
