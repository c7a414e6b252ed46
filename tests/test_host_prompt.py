"""CPU-only checks of the calls on prompts and on the pages' tables: plans, frequencies, and the arguments that are refused before
anything is launched.  No kernel is launched here."""
import ctypes as C
import math
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


def plan(**kw):
    return kvc.PromptPlan(**{**dict(dtype=1, kv_heads=2, q_heads=8, max_batch=3), **kw})


def status_of(call):
    with pytest.raises(kvc.KvcError) as e:
        call()
    return e.value.status


def test_plans(lib):
    for kw in [dict(), dict(dtype=2, rotary_dim=0), dict(rotary_dim=16, layout=kvc.ROTARY_PAIRS), dict(eps=0.0), dict(eps=1e-6, amplitude=1.4),
               dict(frequencies=[-1.0] * 64), dict(q_heads=2), dict(max_batch=65535)]:
        plan(**kw)
    for kw in [dict(dtype=3), dict(dtype=0), dict(layout=2), dict(kv_heads=0), dict(q_heads=7), dict(q_heads=0), dict(max_batch=0),
               dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(amplitude=0.0), dict(amplitude=math.nan), dict(head_dim=0),
               dict(frequencies=[math.nan] * 64), dict(frequencies=[math.inf] * 64), dict(frequencies=[1e10] * 64)]:
        assert status_of(lambda: plan(**kw)) == -1, kw
    for kw in [dict(head_dim=256), dict(rotary_dim=24, frequencies=[1.0] * 12), dict(q_heads=65536), dict(max_batch=65536)]:
        assert status_of(lambda: plan(**kw)) == -2, kw
    with pytest.raises(ValueError):
        plan(frequencies=[1.0] * 63)


def test_null_plans(lib):
    out = C.c_void_p(7)
    assert lib.kvc_prompt_plan(None, 1, C.byref(out)) == -1 and not out.value
    config = kvc.PromptConfig(1, 0, 0, 1, 1, 128, 128, 0.0, 1.0, None)
    assert lib.kvc_prompt_plan(C.byref(config), 1, C.byref(out)) == -1 and not out.value        # (no frequencies)
    config.rotary_dim = 130
    assert lib.kvc_prompt_plan(C.byref(config), 1, C.byref(out)) == -1
    config.rotary_dim = 0
    assert lib.kvc_prompt_plan(C.byref(config), 1, None) == -1
    lib.kvc_prompt_plan_free(None)


def test_frequencies(lib):
    f = kvc.rotary_frequencies(128, 10000.0)
    assert len(f) == 64 and f[0] == 1.0 and f[32] == pytest.approx(0.01, rel=1e-14)
    assert kvc.rotary_frequencies(64, 5e5, kvc.SCALE_LINEAR, 4.0) == pytest.approx([x / 4 for x in kvc.rotary_frequencies(64, 5e5)], rel=1e-14)
    # the base that makes the slowest pair slower by the factor, and leaves the fastest
    g = kvc.rotary_frequencies(128, 10000.0, kvc.SCALE_BASE, 8.0)
    assert g[0] == 1.0 and g[-1] == pytest.approx(f[-1] / 8, rel=1e-12)
    # bands: 8192 tokens; pairs of more than 4 turns unchanged, fewer than 1 divided, between them linear in the turns
    g = kvc.rotary_frequencies(128, 5e5, kvc.SCALE_BANDS, 8.0, 1.0, 4.0, 8192)
    mixed = 0
    for x, y in zip(kvc.rotary_frequencies(128, 5e5), g):
        turns = 8192 * x / (2 * math.pi)
        if turns >= 4:
            assert y == x
        elif turns <= 1:
            assert y == pytest.approx(x / 8, rel=1e-14)
        else:
            t = (turns - 1) / 3
            assert y == pytest.approx(t * x + (1 - t) * x / 8, rel=1e-13)
            mixed += 1
    assert mixed
    # ramp, base 10000, 4096 tokens, 32 and 1 turns: from pair floor(20.94) to ceil(45.03) of 64
    f, g = kvc.rotary_frequencies(128, 10000.0), kvc.rotary_frequencies(128, 10000.0, kvc.SCALE_RAMP, 16.0, 1.0, 32.0, 4096)
    for i, (x, y) in enumerate(zip(f, g)):
        t = min(max((i - 20) / (46 - 20), 0), 1)
        assert y == pytest.approx(t * x / 16 + (1 - t) * x, rel=1e-13), i


def test_frequencies_refused(lib):
    for args in [(0, 1e4), (3, 1e4), (-2, 1e4), (128, 1.0), (128, math.nan), (128, 1e4, 5), (128, 1e4, -1), (128, 1e4, 1, 0.5), (128, 1e4, 1, math.nan),
                 (2, 1e4, 2, 2.0), (128, 1e4, 3, 2.0, 4.0, 1.0), (128, 1e4, 3, 2.0, 0.0, 1.0), (128, 1e4, 4, 2.0, 1.0, math.inf),
                 (128, 1e4, 4, 2.0, 1.0, 32.0, 0)]:
        assert status_of(lambda: kvc.rotary_frequencies(*args)) == -1, args
    assert lib.kvc_rotary_frequencies(128, 1e4, 0, 1.0, 1.0, 4.0, 1, None) == -1


# Device addresses that nothing is read from: the calls below are refused before a launch, or end at the device that is not there.
AT = 1 << 20
ON, OFF = 2 * AT, 3 * AT                    # others


def rows_of(**kw):
    base = dict(q=AT, k=ON, q_out=AT, k_out=ON, q_weight=AT, k_weight=AT, positions=AT, rows=5, q_stride_row=1024, q_stride_head=128,
                k_stride_row=256, k_stride_head=128, q_out_stride_row=1024, q_out_stride_head=128, k_out_stride_row=256, k_out_stride_head=128)
    return kvc.PromptRows(**{**base, **kw})


def test_rotation_refused(lib):
    normed, plain, still = plan(eps=1e-6), plan(), plan(rotary_dim=0)
    call = lambda p, **kw: lib.kvc_prompt_rotate(p._h if p else None, C.byref(rows_of(**kw)), None)            # noqa: E731
    assert lib.kvc_prompt_rotate(plain._h, None, None) == -1 and call(None) == -1
    for kw in [dict(rows=-1), dict(q_out=None), dict(k_out=None), dict(q_weight=None), dict(k_weight=None), dict(positions=None), dict(q=AT + 8),
               dict(k=AT + 2), dict(q_out=AT + 4), dict(k_out=AT + 8), dict(q_weight=AT + 2), dict(positions=AT + 2), dict(q_stride_row=1020),
               dict(k_stride_head=4), dict(q_out_stride_head=129), dict(k_out_stride_row=-4),
               # in place with other strides, over the other input, into one tensor
               dict(q_out_stride_row=2048), dict(q_out_stride_head=256), dict(k_stride_row=512), dict(q_out=ON), dict(k_out=AT), dict(q_out=OFF, k_out=OFF)]:
        assert call(normed, **kw) == -1, kw
    assert call(normed, rows=1 << 31) == -3
    # nothing to do
    assert call(normed, rows=0) == 0 and call(plain, q=None, k=None) == 0
    if not torch.cuda.is_available():
        for p, kw in [(plain, dict(q_weight=None, k_weight=None)), (still, dict(positions=None)), (normed, dict(q=None, q_out=None, q_weight=None)),
                      (normed, dict(k=None, k_out=None, k_weight=None)), (plain, dict(q_stride_row=-1024, q_out_stride_row=-1024)),
                      (plain, dict(q_out=OFF, q_out_stride_row=2048)), (plain, dict(rows=1, q_out_stride_row=2048))]:
            assert call(p, **kw) == -6, kw


def test_attention_refused(lib):
    p = plan()
    base = dict(q=AT, k=AT, v=AT, out=ON, lse=None, rows=9, q_stride_row=1024, q_stride_head=128, k_stride_row=256, k_stride_head=128,
                v_stride_row=256, v_stride_head=128, out_stride_row=1024, out_stride_head=128, scale=0.1)

    def call(n=2, max_rows=9, start=AT, status=AT, plan=p, **kw):
        return lib.kvc_prompt_attend(plan._h if plan else None, C.byref(kvc.PromptSequences(n, max_rows, start)),
                                     C.byref(kvc.PromptHeads(**{**base, **kw})), status, None)
    assert call(plan=None) == -1
    assert lib.kvc_prompt_attend(p._h, None, C.byref(kvc.PromptHeads(**base)), AT, None) == -1
    assert lib.kvc_prompt_attend(p._h, C.byref(kvc.PromptSequences(1, 1, AT)), None, AT, None) == -1
    for kw in [dict(n=-1), dict(max_rows=-1), dict(rows=-1), dict(start=None), dict(status=None), dict(q=None), dict(k=None), dict(v=None),
               dict(out=None), dict(start=AT + 2), dict(status=AT + 1), dict(q=AT + 8), dict(k=AT + 8), dict(v=AT + 8), dict(out=AT + 8), dict(lse=AT + 2),
               dict(q_stride_row=1), dict(k_stride_head=12), dict(v_stride_row=2), dict(out_stride_head=4), dict(scale=math.nan),
               dict(scale=math.inf), dict(scale=-2e38), dict(scale=1e-38), dict(scale=-1e-44),
               # into keys or values; in place with other strides
               dict(q=OFF, k=ON), dict(q=OFF, v=ON), dict(q=ON, out_stride_row=2048), dict(q=ON, q_stride_head=256)]:
        assert call(**kw) == -1, kw
    assert call(n=4) == -3 and call(rows=(1 << 28) + 1) == -3
    for kw in [dict(k_stride_row=-256), dict(v_stride_row=-8), dict(k_stride_row=(1 << 24) + 8), dict(v_stride_row=1 << 40)]:
        assert call(**kw) == -2, kw
    assert call(n=0, start=None) == 0 and call(max_rows=0, q=None) == 0
    if not torch.cuda.is_available():
        assert call() == -6 and call(scale=0.0, lse=AT + 4) == -6 and call(q=ON) == -6 and call(q=ON, rows=1, q_stride_row=0) == -6 and call(k_stride_row=0, v_stride_row=1 << 24, q_stride_row=-1024) == -6 and call(rows=0, q=None, k=None, v=None, out=None) == -6


def test_block_rows(lib):
    """Few rows: 64, shared by two sets of waves where they are long; many: 128; long ones: 192."""
    p = plan(kv_heads=8, q_heads=64, max_batch=300)
    assert p.block_rows(1, 37, 37) == (64, 4) and p.block_rows(200, 30, 6000) == (64, 4)
    few = plan(kv_heads=8, q_heads=32)
    assert few.block_rows(1, 512, 512) == few.block_rows(1, 1024, 1024) == (64, 8)
    assert p.block_rows(1, 2048, 2048)[0] == 128 and p.block_rows(1, 32768, 32768) == (192, 4)
    one = plan(kv_heads=1, q_heads=1)
    assert one.block_rows(1, 8192, 8192) == (64, 8)
    # (a bound beyond the tensors' rows means no more than those)
    assert few.block_rows(1, 1 << 30, 1024) == (64, 8)
    for args in ((0, 5, 5), (301, 5, 5), (1, 0, 5), (1, 5, 0), (-1, 5, 5), (1, 5, (1 << 28) + 1)):
        assert p.block_rows(*args) == (0, 0), args
    waves = C.c_int32(7)
    assert lib.kvc_prompt_block_rows(None, 1, 5, 5, C.byref(waves)) == 0 and waves.value == 0
    assert lib.kvc_prompt_block_rows(p._h, 1, 37, 37, None) == 64


def test_advance_refused(lib):
    p = kvc.CachePlan(1, 2, 8, block_tokens=32, max_tokens=1000, max_batch=6000)
    base = dict(n=3, max_new=9, max_tokens=1000, rows=20, held=AT, kept=None, fresh=AT, free_pages=AT, block_table=AT, table_stride=32, new_start=ON,
                tokens=OFF, positions=4 * AT, slots=5 * AT, num_pages=50)

    def call(plan=p, status=AT, **kw):
        return lib.kvc_cache_advance(plan._h if plan else None, C.byref(kvc.CacheStep(**{**base, **kw})), status, None)
    assert call(plan=None) == -1 and lib.kvc_cache_advance(p._h, None, AT, None) == -1
    for kw in [dict(n=-1), dict(max_new=-1), dict(max_tokens=-1), dict(rows=-1), dict(num_pages=-1), dict(table_stride=31), dict(held=None),
               dict(free_pages=None), dict(block_table=None), dict(new_start=None), dict(tokens=None), dict(status=None), dict(held=AT + 2),
               dict(kept=AT + 1), dict(fresh=AT + 2), dict(free_pages=AT + 2), dict(block_table=AT + 2), dict(new_start=AT + 2), dict(tokens=AT + 2),
               dict(positions=AT + 2), dict(slots=AT + 4), dict(status=AT + 2),
               # written while others read them
               dict(tokens=AT), dict(new_start=AT), dict(positions=AT), dict(slots=AT), dict(kept=OFF), dict(kept=ON), dict(tokens=ON)]:
        assert call(**kw) == -1, kw
    assert call(n=4097) == -3 and call(n=6001) == -3 and call(max_tokens=1001) == -3 and call(rows=1 << 31) == -3
    assert call(n=0, held=None) == 0
    if not torch.cuda.is_available():
        assert call() == -6 and call(kept=AT, fresh=None, positions=None, slots=None, rows=0) == -6


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_tensors_in_host_memory_are_refused(lib):
    half = lambda *shape: torch.zeros(*shape, dtype=torch.float16)                          # noqa: E731
    prompt = kvc.Prompt(plan(), "cpu")
    with pytest.raises(ValueError):
        prompt.rotate(half(2, 8, 128), half(2, 2, 128), i32(0, 1))
    with pytest.raises(ValueError):
        prompt.attend(kvc.PromptBatch(i32(0, 2), 2), half(2, 8, 128), half(2, 2, 128), half(2, 2, 128), half(2, 8, 128), 0.1)
    pages = kvc.CachePages(kvc.CachePlan(1, 2, 8, max_tokens=100, max_batch=2), 7, 2, "cpu")
    assert pages.free_count.item() == 7 and pages.free_pages.tolist() == [6, 5, 4, 3, 2, 1, 0] and pages.table.shape == (2, 7)
    with pytest.raises(ValueError):
        pages.advance(i32(0, 0, 0), i32(0, 0), fresh=i32(1, 1), max_new=1)
    with pytest.raises(ValueError):
        pages.set_free(torch.zeros(8, dtype=torch.int32))


def test_shapes_are_checked(lib, monkeypatch):
    """Tensors that say that they are where the calls want them; none of these calls reaches the library."""
    prompt = kvc.Prompt(plan(eps=1e-6), "cpu")
    prompt._device = -1                      # (what a tensor in host memory says)
    half = lambda *shape: torch.zeros(*shape, dtype=torch.float16)                          # noqa: E731
    q, k, w, p = half(3, 8, 128), half(3, 2, 128), half(128), i32(0, 1, 2)
    monkeypatch.setattr(prompt, "_rotate", lambda *a: pytest.fail("reached"))
    monkeypatch.setattr(prompt, "_attend", lambda *a: pytest.fail("reached"))
    for args in [(q, k[:2], p), (q, k, p[:2]), (q, k, p.long()), (q.float(), k, p), (k, k, p), (q, q, p), (q, k, p, q[:2]), (q, k, p, q, k[:, :1]),
                 (half(0, 8, 128), k, p)]:
        with pytest.raises(ValueError):
            prompt.rotate(*args, **dict(q_weight=w, k_weight=w))
    for weights in [dict(), dict(q_weight=w), dict(q_weight=w, k_weight=w.float()), dict(q_weight=w, k_weight=w[:64])]:
        with pytest.raises(ValueError):
            prompt.rotate(q, k, p, **weights)
    batch = kvc.PromptBatch(i32(0, 3), 3)
    for args in [(q, k[:2], k, q), (q, k, k[:2], q), (q, k, k, q[:2]), (q, q, k, q), (q.bfloat16(), k, k, q)]:
        with pytest.raises(ValueError):
            prompt.attend(batch, *args, 0.1)
    for lse in (torch.zeros(3, 7), torch.zeros(3, 8, dtype=torch.float64), torch.zeros(8, 3).T):
        with pytest.raises(ValueError):
            prompt.attend(batch, q, k, k, q, 0.1, lse)
    for start in (i32(0, 3).long(), i32(0, 3).reshape(1, 2), i32(0, 9, 3)[::2], torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError):
            kvc.PromptBatch(start, 3)
    pages = kvc.CachePages(kvc.CachePlan(1, 2, 8, max_tokens=100, max_batch=2), 7, 2, "cpu")
    pages._device = -1
    monkeypatch.setattr(pages, "_advance", lambda *a: pytest.fail("reached"))
    a, b = i32(0, 0, 0), i32(0, 0)
    for args, kw in [((b, b), {}), ((a, a), {}), ((a, b.long()), {}), ((a, b), dict(kept=a)), ((a, b), dict(fresh=b.long())),
                     ((a, b), dict(positions=i32(1, 2), slots=torch.zeros(3, dtype=torch.int64))), ((a, b), dict(positions=torch.zeros(3))),
                     ((a, b), dict(slots=i32(1))), ((a, b), dict(positions=i32(1, 2), rows=3)), ((a, b), dict(positions=i32(1, 2, 3)[::2]))]:
        with pytest.raises(ValueError):
            pages.advance(*args, **kw)


def test_the_calls_go_to_their_device(lib, monkeypatch):
    """Two devices, the first of which is current: a call makes its own the current one while it launches."""
    at, seen = [0], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            at.append(self.device)

        def __exit__(self, *_):
            at.pop()

    class OnSecondDevice(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1

    class Recorder:
        def __getattr__(self, name):
            if name not in ("kvc_prompt_rotate", "kvc_prompt_attend", "kvc_cache_advance"):
                return getattr(lib, name)

            def call(*args):
                seen.append((name, at[-1]))
                return 0
            return call

    zeros, full = torch.zeros, torch.full
    second = lambda *a, device=None, **kw: zeros(*a, **kw).as_subclass(OnSecondDevice)       # noqa: E731
    monkeypatch.setattr(torch, "zeros", second)
    monkeypatch.setattr(torch, "full", lambda *a, device=None, **kw: full(*a, **kw).as_subclass(OnSecondDevice))
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    cache_plan, prompt_plan = kvc.CachePlan(1, 2, 8, max_tokens=100, max_batch=2), plan()
    monkeypatch.setattr(kvc, "_lib", Recorder())
    prompt, pages = kvc.Prompt(prompt_plan, "cuda:1"), kvc.CachePages(cache_plan, 7, 2, "cuda:1")
    words = lambda *v: i32(*v).as_subclass(OnSecondDevice)                                   # noqa: E731
    q, k = second(2, 8, 128, dtype=torch.float16), second(2, 2, 128, dtype=torch.float16)
    prompt.rotate(q, k, words(0, 1))
    prompt.attend(kvc.PromptBatch(words(0, 2), 2), q, k, k, q, 0.1)
    pages.advance(words(0, 0, 0), words(0, 0))
    assert seen == [("kvc_prompt_rotate", 1), ("kvc_prompt_attend", 1), ("kvc_cache_advance", 1)] and at == [0]


def test_packed_arguments():
    """The bytes that the calls are given are those of the structures."""
    for structure, pack in ((kvc.CacheStep, kvc._pack_step), (kvc.PromptRows, kvc._pack_rows), (kvc.PromptHeads, kvc._pack_heads)):
        values = [2.5 if t is C.c_float else (i + 1) * 0x10203 * (-1 if t is C.c_int64 else 1) for i, (_, t) in enumerate(structure._fields_)]
        made = structure.from_buffer_copy(pack(*values))
        assert [getattr(made, name) for name, _ in structure._fields_] == values
