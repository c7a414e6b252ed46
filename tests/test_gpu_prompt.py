"""GPU tests (run with -m gpu): attention over whole prompts against 64-bit values."""
import math

import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, attention, check_attention, heads, i32, own_type, stream, typed

pytestmark = pytest.mark.gpu
SCALE = DIM ** -0.5


class Case:
    def __init__(self, lengths, kv_heads=2, per_kv=3, bf16=False, seed=0, fused=False, before=0, behind=0, spread=1.0, max_batch=None):
        self.lengths, self.bf16, self.before = lengths, bf16, before
        self.starts = (before + np.concatenate([[0], np.cumsum(lengths)])).tolist()
        rows = self.starts[-1] + behind
        self.q, self.k, self.v = heads(rows, kv_heads, per_kv, bf16, seed, fused, spread)
        self.start = i32(*self.starts)
        self.prompt = kvc.Prompt(kvc.PromptPlan(own_type(bf16), kv_heads, kv_heads * per_kv, max_batch=max_batch or len(lengths)))
        self.batch = kvc.PromptBatch(self.start, max(max(lengths), 1))
        self.out = torch.full(self.q.shape, 77.0, dtype=typed(bf16), device=DEVICE)
        self.lse = torch.full(self.q.shape[:2], 77.0, dtype=torch.float32, device=DEVICE)

    def run(self, scale=SCALE, **kw):
        self.prompt.attend(self.batch, self.q, self.k, self.v, self.out, scale, self.lse, stream(), **kw)
        return self

    def check(self, scale=SCALE, only=None, status=None):
        for s, (a, b) in enumerate(zip(self.starts, self.starts[1:])):
            if b > a and (only is None or s in only):
                check_attention(self.out[a:b], self.lse[a:b], self.q[a:b], self.k[a:b], self.v[a:b], scale, self.bf16)
        a, b = self.starts[0], self.starts[-1]
        for x in (self.out, self.lse):
            assert (x[:a] == 77).all() and (x[b:] == 77).all()
        if status is None:
            assert not self.prompt.status.any()


LENGTHS = [[1], [2], [31, 32, 33], [15, 16, 17, 1], [63, 64, 65], [127, 128, 129, 0], [0, 191, 192, 193], [255, 256, 257], [0], [511, 3], [700, 0, 0, 41, 513]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("bf16", [False, True])
def test_lengths(lengths, bf16):
    Case(lengths, bf16=bf16, seed=sum(lengths), fused=len(lengths) % 2 == 0, before=5 * (len(lengths) > 2), behind=3).run().check()


@pytest.mark.parametrize("kv_heads,per_kv", [(1, 1), (1, 8), (8, 1), (8, 8), (3, 5), (4, 16), (10, 2)])
@pytest.mark.parametrize("bf16", [False, True])
def test_heads(kv_heads, per_kv, bf16):
    Case([130, 77], kv_heads, per_kv, bf16, seed=kv_heads, fused=bf16).run().check()


def test_many_sequences():
    """More sequences than are sorted by their lengths, empty ones among them."""
    g = np.random.default_rng(5)
    for n in (63, 64, 65, 255, 256, 257, 512, 700, 1500):
        lengths = g.integers(0, 9, n).tolist()
        lengths[n // 2], lengths[-1], lengths[0] = 150, 20, 70
        Case(lengths, 1, 2, n % 2 == 0, seed=n, behind=1).run().check()


@pytest.mark.parametrize("bf16", [False, True])
def test_ragged_order(bf16):
    """Sequences whose blocks are mixed, longest first."""
    Case([300, 1, 640, 128, 129, 0, 384, 2, 900, 64], 2, 2, bf16, seed=9).run().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.07, 3.0, 1e-30])
def test_scales(scale, bf16):
    Case([140, 30], bf16=bf16, seed=3).run(scale).check(scale)


@pytest.mark.parametrize("bf16", [False, True])
def test_rising_and_falling_scores(bf16):
    """Maxima that grow by a lot and by little from tile to tile, and scores far below the first one."""
    for rising in (1, -1):
        c = Case([420], 1, 2, bf16, seed=4)
        t = torch.linspace(0.2, 3.0, 420, device=DEVICE) if rising > 0 else torch.linspace(3.0, 0.2, 420, device=DEVICE)
        c.q[:] = 1.0
        c.k[:] = (t[:, None, None] * 10).to(c.k.dtype)
        c.run().check()


def test_weights_far_below_the_largest():
    """fp16: 2000 tokens of weight 2^-24 each beside one of weight 1 are no nothing."""
    c = Case([2100], 1, 1, False, seed=6)
    c.q[:], c.k[:], c.v[:] = 0, 0, 0
    c.q[:, :, 0] = 1
    c.k[0, :, 0] = 24 * math.log(2.0)        # score of token 0, with scale 1; the others' is 0
    c.v[1:] = 1024.0
    c.run(1.0).check(1.0)
    assert c.out[-1].min() > 0.1


@pytest.mark.parametrize("value", [3.3e38, -1e37, 1e30, 1e-30])
def test_large_and_small_values(value):
    """bf16: sums of thousands of the largest values, and of small ones, stay inside 32 bits; so do scores that rise."""
    for rising in (False, True):
        c = Case([5000], 1, 1, True, seed=6)
        c.q[:] = 1
        c.k[:] = 0 if not rising else (torch.linspace(0.0, 0.5, 5000, device=DEVICE)[:, None, None]).bfloat16()
        c.v[:] = value
        c.run()
        assert ((c.out.double() / c.v.double() - 1).abs() <= 2.0 ** -7).all()
        c.check()


@pytest.mark.parametrize("bf16", [False, True])
def test_equal_values_give_themselves(bf16):
    """A mean of equal numbers: weights and their sum have the same roundings but for half a step of each."""
    c = Case([333], 2, 2, bf16, seed=8)
    c.v[:] = 3.0
    c.run().check()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("at", [0, 5, 63, 64, 100, 199])
def test_what_is_not_seen_does_not_matter(bad, bf16, at):
    """A key and a value that are no finite numbers: the rows before them have the same bits as without them, the rows from there on no finite
    results (key) or none in the value's channel."""
    clean = Case([70, 200, 60], 2, 2, bf16, seed=at).run()
    clean.check()
    a = 70 + at
    for what in ("k", "v", "both"):
        c = Case([70, 200, 60], 2, 2, bf16, seed=at)
        if what != "v":
            c.k[a, 1, 7] = bad
        if what != "k":
            c.v[a, 1, 40] = bad
        c.run()
        assert not c.prompt.status.any()
        same = torch.ones(c.out.shape, dtype=torch.bool, device=DEVICE)
        rows = slice(a, 270)
        if what != "v":
            # (a score of -infinity is a weight of zero: that row's result is finite)
            if math.isnan(bad):
                assert c.out[rows, 2:].isnan().all() and c.lse[rows, 2:].isnan().all()
            same[rows, 2:] = False
        else:
            assert not c.out[rows, 2:, 40].isfinite().any()
            same[rows, 2:, 40] = False
        # (the block is done again with the same steps)
        assert torch.equal(c.out[same], clean.out[same])
        if what == "v":
            assert torch.equal(c.lse, clean.lse)


@pytest.mark.parametrize("bf16", [False, True])
def test_minus_infinite_scores_weigh_nothing(bf16):
    """Keys that make a score of -infinity: as if the token were not there, also where it comes first."""
    c = Case([150], 1, 1, bf16, seed=2)
    c.q[:] = c.q.abs() + 0.1
    c.k[:70] = -math.inf
    c.v[:70] = 50.0
    c.run()
    want, want_lse, _, _ = attention(c.q, c.k, c.v, SCALE)
    assert c.out[:70].isnan().all()          # nothing to weigh
    assert ((c.out[70:].double() - want[70:]).abs() <= 0.02).all() and ((c.lse[70:] - want_lse[70:]).abs() < 1e-3).all()


@pytest.mark.parametrize("bf16", [False, True])
def test_neighbours_may_hold_anything(bf16):
    """Rows before, between and behind hold NaN and infinities."""
    clean = Case([50, 130, 70], 2, 2, bf16, seed=1, before=9, behind=200).run()
    c = Case([50, 130, 70], 2, 2, bf16, seed=1, before=9, behind=200)
    for x in (c.q, c.k, c.v):
        x[:59], x[59 + 130:] = math.nan, math.inf
        x[9 + 50 + 130 + 70:] = -math.inf
    c.run()
    assert torch.equal(c.out[59:189], clean.out[59:189]) and torch.equal(c.lse[59:189], clean.lse[59:189])
    assert (c.out[-200:] == 77).all() and (c.out[:9] == 77).all()


def test_queries_that_are_no_numbers():
    """They spoil their own row and head only."""
    clean, c = Case([180], 2, 2, seed=1).run(), Case([180], 2, 2, seed=1)
    c.q[33, 1, 5], c.q[90, 3, 0] = math.nan, math.inf
    c.run()
    same = torch.ones(180, 4, dtype=torch.bool, device=DEVICE)
    same[33, 1] = same[90, 3] = False
    assert torch.equal(c.out[same], clean.out[same]) and c.out[33, 1].isnan().all() and c.out[90, 3].isnan().all()
    assert c.lse[33, 1].isnan()


@pytest.mark.parametrize("starts,bad", [([-3, 20, 60], [0]), ([0, 60, 40, 90], [1]), ([0, 30, 5000], [1]), ([0, 10, 200], [1]), ([0, 100, -2 ** 31, 90], [1, 2]),
                                        ([2 ** 31 - 1, 0, 60], [0])])
def test_sequences_that_do_not_fit(starts, bad):
    """They are left out and reported; the others are done.  100 rows, 150 at most."""
    q, k, v = heads(210, 1, 2, False, 3)
    out, n = torch.full_like(q, 77.0), len(starts) - 1
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, 1, 2, max_batch=n))
    prompt.attend(kvc.PromptBatch(i32(*starts), 150), q, k, v, out, SCALE, None, stream())
    assert prompt.status.tolist() == [kvc.DEV_BAD_ROW if s in bad else 0 for s in range(n)]
    for s in range(n):
        if s not in bad:
            a, b = starts[s], starts[s + 1]
            # (rows that a second sequence has too, where starts descend, get the result of one of them)
            one = torch.tensor([r - a for r in range(a, b) if sum(starts[i] <= r < starts[i + 1] for i in range(n) if i not in bad) == 1],
                               device=DEVICE)
            check_attention(out[a:b], None, q[a:b], k[a:b], v[a:b], SCALE, False, one)
    if bad == [0]:
        assert starts[0] < 0 and (out[60:] == 77).all() or starts[0] > 0


def test_overlapping_sequences_are_all_done():
    """Starts that go back now and then give more blocks than the rows have."""
    n = 300
    starts = [0, 100] * n + [0]
    q, k, v = heads(100, 1, 1, True, 3)
    out, lse = torch.full_like(q, 77.0), torch.zeros(100, 1, device=DEVICE)
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.BF16, 1, 1, max_batch=2 * n))
    prompt.attend(kvc.PromptBatch(i32(*starts), 100), q, k, v, out, SCALE, lse, stream())
    assert prompt.status.tolist() == [0, kvc.DEV_BAD_ROW] * n
    check_attention(out, lse, q, k, v, SCALE, True)


def test_no_rows():
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, 1, 2, max_batch=2))
    none = torch.zeros(0, 2, DIM, dtype=torch.float16, device=DEVICE)
    prompt.attend(kvc.PromptBatch(i32(0, 0, 0), 5), none, none[:, :1], none[:, :1], none, SCALE, None, stream())
    prompt.attend(kvc.PromptBatch(i32(0), 5), none, none[:, :1], none[:, :1], none, SCALE, None, stream())
    assert not prompt.status.any()
    prompt.attend(kvc.PromptBatch(i32(0, 1, 1), 5), none, none[:, :1], none[:, :1], none, SCALE, None, stream())
    assert prompt.status.tolist() == [kvc.DEV_BAD_ROW] * 2               # (the second starts behind the rows)


@pytest.mark.parametrize("bf16", [False, True])
def test_in_place_and_without_lse(bf16):
    c = Case([200, 65], 2, 4, bf16, seed=4, fused=True).run()
    q = c.q.clone()
    view = torch.empty(c.q.shape[0], 3 * 8, DIM, dtype=c.q.dtype, device=DEVICE)[:, 4:12]
    view.copy_(q)
    c.prompt.attend(c.batch, view, c.k, c.v, view, SCALE, None, stream())
    assert torch.equal(view, c.out)


def test_layouts():
    """Heads before rows, one row, one head."""
    c = Case([90], 2, 2, True, seed=2).run()
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.q, c.k, c.v)]
    out = torch.empty(4, 90, DIM, dtype=c.q.dtype, device=DEVICE).transpose(0, 1)
    c.prompt.attend(c.batch, *turned, out, SCALE, None, stream())
    assert torch.equal(out, c.out)
    # broadcast keys: one row's stride of zero
    k = c.k[:1].expand(90, 2, DIM)
    c.prompt.attend(c.batch, c.q, k, c.v, out, SCALE, None, stream())
    check_attention(out, None, c.q, k, c.v, SCALE, True)


@pytest.mark.parametrize("bf16", [False, True])
def test_packed_is_as_alone(bf16):
    """Equal inputs and bounds give equal bits: again, and each sequence in a call of its own."""
    c = Case([300, 77, 1, 520], 2, 2, bf16, seed=5).run()
    first = c.out.clone(), c.lse.clone()
    c.run()
    assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])
    block = c.prompt.plan.block_rows(4, 520, 898)
    for a, b in zip(c.starts, c.starts[1:]):
        out = torch.full_like(c.q, 77.0)
        assert c.prompt.plan.block_rows(1, 520, 898) == block
        c.prompt.attend(kvc.PromptBatch(i32(a, b), 520), c.q, c.k, c.v, out, SCALE, None, stream())
        assert torch.equal(out[a:b], c.out[a:b]) and (out[:a] == 77).all() and (out[b:] == 77).all()


def test_bounds_above_the_lengths():
    """max_rows and max_batch far above what there is, as a captured step has them."""
    c = Case([130, 40], 2, 2, seed=6)
    c.batch = kvc.PromptBatch(c.start, 1 << 20)
    c.run().check()


@pytest.mark.parametrize("bf16,kv_heads,per_kv,rows", [(False, 1, 2, 20011), (True, 8, 1, 4099), (True, 1, 8, 2500)])
def test_long(bf16, kv_heads, per_kv, rows):
    c = Case([rows, 1200], kv_heads, per_kv, bf16, seed=7).run()
    some = torch.tensor(sorted({0, 1, 127, 128, rows // 2, rows - 2, rows - 1} | set(np.random.default_rng(1).integers(0, rows, 60).tolist())), device=DEVICE)
    check_attention(c.out[:rows], c.lse[:rows], c.q[:rows], c.k[:rows], c.v[:rows], SCALE, bf16, some)


def test_offsets_beyond_32_bits():
    """Rows 200 kB apart: 23000 of them are more than 2^32 bytes, and 2^31 elements."""
    rows, stride = 23000, 100000
    x = torch.empty(rows, stride, dtype=torch.float16, device=DEVICE)
    q, k, v, out = (x[:, i * DIM: (i + 1) * DIM].unflatten(1, (1, DIM)) for i in range(4))
    g = torch.Generator(device=DEVICE).manual_seed(3)
    for y in (q, k, v):
        y.copy_(torch.randn(y.shape, generator=g, device=DEVICE))
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, 1, 1))
    prompt.attend(kvc.PromptBatch(i32(0, rows), rows), q, k, v, out, SCALE, None, stream())
    some = torch.tensor([0, 63, 64, 10000, 21474, 21475, 21476, 22000, rows - 1], device=DEVICE)
    check_attention(out, None, q, k, v, SCALE, False, some)


def test_captured_and_replayed():
    """Lengths that change between replays, with eager calls in between."""
    c = Case([100, 250, 7], 2, 2, True, seed=8, behind=150)
    c.batch = kvc.PromptBatch(c.start, 400)
    c.run()                                  # (loads what has to be loaded)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for lengths in ([100, 250, 7], [300, 0, 200], [1, 1, 1], [7, 400, 99]):
        starts = np.concatenate([[0], np.cumsum(lengths)]).tolist()
        c.start.copy_(i32(*starts))
        c.out.fill_(77.0)
        c.lse.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        out, lse = c.out.clone(), c.lse.clone()
        c.starts = starts
        c.check()
        c.out.fill_(77.0)
        c.lse.fill_(77.0)
        c.run()
        assert torch.equal(out, c.out) and torch.equal(lse, c.lse)


def test_two_streams():
    """Two calls at once on streams of their own."""
    cases = [Case([700, 30], 2, 4, bf16, seed=9) for bf16 in (False, True)]
    torch.cuda.synchronize()
    for c, s in zip(cases, (torch.cuda.Stream(), torch.cuda.Stream())):
        for _ in range(3):
            c.prompt.attend(c.batch, c.q, c.k, c.v, c.out, SCALE, c.lse, s.cuda_stream)
    torch.cuda.synchronize()
    for c in cases:
        c.check()
