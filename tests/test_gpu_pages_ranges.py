"""GPU tests (run with -m gpu): the sequences' tables where the numbers of new rows leave 32 bits."""
import pytest

from paper_2605_13734_amd import kvc
from prompt_util import i32, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("last", [-1, 0, 1])
def test_rows_beyond_the_largest_number(last):
    """Without room of its own for the rows a call has 2^31 - 1 of them: what crosses that is left out and reported, and keeps what it holds."""
    big, bt = 1 << 29, 4096
    plan = kvc.CachePlan(kvc.F16, 1, 1, block_tokens=bt, max_tokens=big + bt, max_batch=7)
    p = kvc.CachePages(plan, 600000, 7)
    start, tokens = i32(*[0] * 8), i32(*[0] * 7)
    p.advance(start, tokens, None, i32(0, 3, 0, 0, 0, 0, 9), 9, stream=stream())
    assert tokens.tolist() == [0, 3, 0, 0, 0, 0, 9] and p.free[0] == 600000 - 2
    fresh = [big, big, big, big - 1 + last, 1, 0, 2]                     # (the fourth ends at 2^31 - 1 + last)
    p.advance(start, tokens, None, i32(*fresh), big, stream=stream())
    bad, top = kvc.DEV_BAD_ROW, 2 ** 31 - 1
    over = [sum(fresh[: s + 1]) > top for s in range(7)]
    held = [h if o else h + f for h, f, o in zip([0, 3, 0, 0, 0, 0, 9], fresh, over)]
    assert p.status.tolist() == [bad * o for o in over]
    assert tokens.tolist() == [-1 if o else h for h, o in zip(held, over)] and p.held.tolist() == held
    assert start.tolist() == [min(sum(fresh[:s]), top) for s in range(8)]
    assert p.free[0] == 600000 - sum((h + bt - 1) // bt for h in held)
