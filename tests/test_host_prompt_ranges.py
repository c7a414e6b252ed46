"""CPU-only checks of the calls on prompts and on the pages' tables: results whose parts would share a place, and sizes at the ends of what is
taken.  No kernel is launched here."""
import ctypes as C
import itertools

import pytest
import torch

from paper_2605_13734_amd import kvc

AT, ON = 1 << 20, 1 << 21                   # device addresses that nothing is read from
OK, ARG, CAPACITY, DEVICE = 0, -1, -3, -6


def rotate(q_heads, kv_heads, rows, q=None, k=None):
    """The status of a rotation into results with these (row, head) strides."""
    plan = kvc.PromptPlan(kvc.F16, kv_heads, q_heads)
    a = dict(q=AT if q else None, q_out=ON, k=AT if k else None, k_out=ON + AT, positions=AT, rows=rows, q_stride_row=0, q_stride_head=0, k_stride_row=0,
             k_stride_head=0)
    for name, strides in (("q", q), ("k", k)):
        a[name + "_out_stride_row"], a[name + "_out_stride_head"] = strides or (0, 0)
    return kvc.load().kvc_prompt_rotate(plan._h, C.byref(kvc.PromptRows(**a)), None)


def attend(q_heads, rows, strides, most=None):
    plan = kvc.PromptPlan(kvc.F16, 1, q_heads)
    heads = kvc.PromptHeads(q=AT, k=AT, v=AT, out=ON, rows=rows, q_stride_row=0, q_stride_head=0, k_stride_row=0, k_stride_head=0, v_stride_row=0,
                            v_stride_head=0, out_stride_row=strides[0], out_stride_head=strides[1], scale=0.1)
    return kvc.load().kvc_prompt_attend(plan._h, C.byref(kvc.PromptSequences(1, most or rows, AT)), C.byref(heads), AT, None)


def share(heads, rows, row, head):
    """Whether two heads of a result have a place in common."""
    at = sorted(r * row + h * head for r in range(rows) for h in range(heads))
    return any(b - a < 128 for a, b in zip(at, at[1:]))


STRIDES = [0, 8, 64, 120, 128, 136, 192, 256, 320, 384, 512, 640, 1000, 1024, 1280, 2048, -128, -120, -384, 1 << 40, -(1 << 62)]


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are taken end at the device that is not there")
@pytest.mark.parametrize("heads,rows", [(1, 1), (1, 5), (5, 1), (2, 2), (3, 8), (8, 3), (16, 40)])
def test_results_whose_heads_share_places_are_refused(heads, rows):
    seen = set()
    for strides in itertools.product(STRIDES, STRIDES):
        want = ARG if share(heads, rows, *strides) else DEVICE
        assert rotate(heads, heads, rows, q=strides) == rotate(heads, heads, rows, k=strides) == attend(heads, rows, strides) == want, strides
        seen.add(want)
    assert len(seen) == 2 or heads == rows == 1
    assert attend(heads, 0, (0, 0)) == OK and attend(heads, 0, (0, 0), 5) == DEVICE            # (no rows: nothing is written)


@pytest.mark.parametrize("bad", [lambda x: x[:1].expand(4, 2, 128), lambda x: x[:, :1].expand(4, 2, 128)], ids=["rows", "heads"])
def test_expanded_results_are_refused(bad):
    """Tensors that say that they are where the calls want them."""
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, 2, 2), "cpu")
    prompt._device = -1
    x, y, at = torch.zeros(4, 2, 128, dtype=torch.float16), torch.ones(4, 2, 128, dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: prompt.rotate(x, None, at, bad(y)), lambda: prompt.rotate(None, x, at, None, bad(y)), lambda: prompt.rotate(bad(y), None, at),
                 lambda: prompt.attend(kvc.PromptBatch(torch.zeros(2, dtype=torch.int32), 4), x, x.clone(), x.clone(), bad(y), 0.1)):
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.status == ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are taken end at the device that is not there")
def test_all_rows_that_are_documented_are_taken():
    for heads in (1, 16, 64, 1024):
        stride = (heads * 128, 128)
        assert rotate(heads, 1, 1 << 28, q=stride) == rotate(heads, heads, 1 << 28, q=stride, k=stride) == attend(heads, 1 << 28, stride) == DEVICE
        assert rotate(heads, 1, (1 << 28) + 1, q=stride) == attend(heads, (1 << 28) + 1, stride) == CAPACITY


def test_new_tokens_need_their_bound(monkeypatch):
    """Without it every sequence that gets a token would be left out."""
    pages = kvc.CachePages(kvc.CachePlan(1, 2, 8, max_tokens=100, max_batch=2), 7, 2, "cpu")
    pages._device, calls = -1, []
    monkeypatch.setattr(pages, "_advance", lambda plan, step, status, stream: calls.append(kvc.CacheStep.from_buffer_copy(step).max_new) or 0)
    start, two = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="max_new"):
        pages.advance(start, two, fresh=two.clone())
    pages.advance(start, two, fresh=two.clone(), max_new=0)
    pages.advance(start, two, fresh=two.clone(), max_new=5)
    pages.advance(start, two)
    assert calls == [0, 5, 0]
