"""GPU tests (run with -m gpu) of the quantised cache: rows against the oracle bit for bit, attention against 64-bit values within
tolerances that follow from its roundings (cache_util.World.check_attention), accepted drafts moved, damaged arguments."""
import itertools

import numpy as np
import pytest
import torch

from cache_util import DIM, World, tree_masks
from paper_2605_13734_amd import kvc

pytestmark = pytest.mark.gpu
SCALE = 1 / np.sqrt(DIM)


def stream():
    return torch.cuda.current_stream().cuda_stream


def read_all(w):
    rows = sum(w.total)
    k = torch.full((rows, w.kv_heads, DIM), 7.0, dtype=w.dtype, device="cuda")
    v = torch.full_like(k, 7.0)
    w.cache.load(w.all_batch(), k, v, stream())
    return k.double().cpu().numpy(), v.double().cpu().numpy()


def check_rows(w, expect=None):
    k, v = read_all(w)
    assert not w.cache.status.any()
    at = 0
    for s, t in enumerate(w.total):
        hk, hv = w.held(s)
        pick = list(range(t)) if expect is None else expect[s]
        want_k, want_v = hk.read_back(w.bf16)[pick], hv.read_back(w.bf16)[pick]
        n = len(pick)
        assert np.array_equal(k[at: at + n], want_k), s
        assert np.array_equal(v[at: at + n], want_v), s
        at += t


@pytest.mark.parametrize("bits_k,bits_v,group", list(itertools.product((4, 8), (4, 8), (32, 64, 128))))
@pytest.mark.parametrize("bf16,transform", [(False, 0), (True, 0), (False, 1), (True, 1)])
def test_rows_match_the_oracle(bits_k, bits_v, group, bf16, transform):
    w = World([0, 5, 33, 16], [37, 1, 0, 16], seed=group + bits_k, bf16=bf16, kv_heads=3, bits_k=bits_k, bits_v=bits_v, group=group,
              block_tokens=16 if group == 32 else 32, transform=transform)
    w.fill()
    check_rows(w)


@pytest.mark.parametrize("heads,block_tokens", [(1, 16), (5, 64), (8, 128)])
def test_row_by_row_is_the_same_as_at_once(heads, block_tokens):
    w = World([0, 0], [70, 41], seed=heads, kv_heads=heads, block_tokens=block_tokens)
    w.fill()
    at_once = w.cache.pages.clone()
    check_rows(w)
    w.cache.pages.fill_(0xff)
    for i in range(70):                                       # sequence 1 stops growing at 41
        new = [1, 1 if i < 41 else 0]
        tokens = torch.tensor([i + 1, min(i + 1, 41)], dtype=torch.int32, device="cuda")
        b = kvc.CacheBatch(w.starts(new), tokens, w.table, 1, 70, w.num_pages)
        pick = [w.k[0][i: i + 1]] + ([w.k[1][i: i + 1]] if new[1] else []), [w.v[0][i: i + 1]] + ([w.v[1][i: i + 1]] if new[1] else [])
        w.cache.store(b, torch.cat(pick[0]).cuda(), torch.cat(pick[1]).cuda(), stream())
    assert torch.equal(at_once, w.cache.pages)


@pytest.mark.parametrize("bf16,transform", [(False, 0), (True, 0), (True, 1)])
def test_extreme_rows(bf16, transform):
    """Zeros, one value, the type's limits, subnormals, infinities and NaN; what stands in one row stays there."""
    w = World([0], [12], seed=3, bf16=bf16, kv_heads=1, bits_k=8, bits_v=4, group=64, transform=transform)
    x = torch.randn(12, 1, DIM)
    x[0] = 0.0
    x[1] = -3.25
    x[2] = 65504.0
    x[3, :, ::2], x[3, :, 1::2] = 65504.0, -65504.0
    x[4] = torch.randn(1, DIM) * 1e-7
    x[5] = -0.0
    x[6, 0, 5] = 1e30 if bf16 else 60000.0
    if not transform:
        x[7, 0, 3], x[7, 0, 4] = float("inf"), float("-inf")
        x[8, 0, 9] = float("nan")
        x[9] = float("nan")
    w.k[0] = w.v[0] = x.to(w.dtype)
    w.fill()
    check_rows(w)


def test_strided_rows_and_other_memory():
    """K and V inside one fused tensor; what lies between their rows and the pages nobody named stay as they are."""
    w = World([3, 40], [19, 6], seed=8, kv_heads=2, per_kv=3, block_tokens=32)
    w.cache.store(w.past_batch(), *w.old_rows(), stream())
    fused = torch.randn(25, 10, DIM, device="cuda").to(w.dtype)
    k, v = w.new_rows()
    fused[:, 6:8], fused[:, 8:10] = k, v
    before = fused.clone()
    w.cache.store(w.batch(), fused[:, 6:8], fused[:, 8:10], stream())
    check_rows(w)
    assert torch.equal(before, fused)
    pages = w.cache.pages[: w.num_pages * w.plan.page_bytes()].reshape(w.num_pages, -1)
    assert (pages[w.free_pages.cuda()] == 0xff).all()
    out = torch.full_like(fused, 5.0)
    w.cache.load(w.batch(), out[:, 1:3], out[:, 4:6], stream())
    rest = [0, 3, 6, 7, 8, 9]
    assert (out[:, rest] == 5.0).all()
    at = 0
    for s in range(2):
        hk, hv = w.held(s)
        n = w.new[s]
        assert np.array_equal(out[at: at + n, 1:3].double().cpu().numpy(), hk.read_back(False)[w.past[s]:])
        assert np.array_equal(out[at: at + n, 4:6].double().cpu().numpy(), hv.read_back(False)[w.past[s]:])
        at += n


def attend(w, masks=None, scale=SCALE, lse=True):
    out = torch.full_like(w.q, float("nan"), device="cuda")
    stat = torch.full(w.q.shape[:2], float("nan"), device="cuda") if lse else None
    w.cache.attend(w.batch(None if masks is None else w.mask_tensor(masks)), w.q.cuda(), out, scale, stat, stream())
    assert not w.cache.status.any()
    w.check_attention(out, stat, scale, masks)
    return out


@pytest.mark.parametrize("bits_k,bits_v,group", list(itertools.product((4, 8), (4, 8), (32, 64, 128))))
@pytest.mark.parametrize("bf16,transform,per_kv", [(False, 0, 4), (True, 0, 5), (False, 1, 16), (True, 1, 8)])
def test_attention_of_single_tokens(bits_k, bits_v, group, bf16, transform, per_kv):
    w = World([0, 15, 130, 611], [1, 1, 1, 1], seed=per_kv, bf16=bf16, per_kv=per_kv, bits_k=bits_k, bits_v=bits_v, group=group,
              transform=transform, block_tokens=16 if bf16 else 64)
    w.fill()
    attend(w)


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 32, 33, 63, 127, 128, 129, 255, 256, 257, 1023, 1025, 4097])
def test_attention_lengths(tokens):
    w = World([tokens - 1], [1], seed=tokens, kv_heads=1, per_kv=7)
    w.fill()
    attend(w)


@pytest.mark.parametrize("new,per_kv", [(2, 4), (5, 3), (16, 1), (9, 8), (33, 1), (17, 8), (64, 2), (65, 4), (131, 1)])
@pytest.mark.parametrize("bf16,transform,group", [(False, 0, 32), (True, 1, 64), (False, 1, 128)])
def test_attention_of_consecutive_tokens(new, per_kv, bf16, transform, group):
    w = World([0, 77, 300], [new, max(new // 2, 1), new], seed=new, bf16=bf16, per_kv=per_kv, transform=transform, group=group, block_tokens=32,
              bits_k=8 if bf16 else 4)
    w.fill()
    attend(w)


@pytest.mark.parametrize("new,past,bits_v", [(1, 0, 4), (7, 20, 4), (16, 129, 8), (63, 1, 4), (64, 500, 4), (65, 64, 8), (100, 31, 4)])
@pytest.mark.parametrize("transform,per_kv", [(0, 4), (1, 8), (0, 1)])
def test_attention_of_trees(new, past, bits_v, transform, per_kv):
    w = World([past, 0, past + 3], [new, (new + 1) // 2, new], seed=new + past, per_kv=per_kv, bits_v=bits_v, transform=transform)
    masks, _ = tree_masks(w.g, w.new)
    w.fill()
    attend(w, masks)


@pytest.mark.parametrize("bits_k,bits_v,group", list(itertools.product((4, 8), (4, 8), (32, 64, 128))))
@pytest.mark.parametrize("bf16,transform", [(False, 0), (True, 0), (False, 1), (True, 1)])
@pytest.mark.parametrize("new", [7, 37])
def test_attention_of_every_kind(bits_k, bits_v, group, bf16, transform, new):
    """Blocks of 32 rows and of 128, each pair of widths, group, type and transform: a tree behind nothing and behind a context that is
    cut, and one token."""
    w = World([0, 900, 45], [new, new, 1], seed=new + group, kv_heads=1, per_kv=4, bf16=bf16, bits_k=bits_k, bits_v=bits_v, group=group,
              transform=transform, block_tokens=32)
    masks, _ = tree_masks(w.g, w.new)
    w.fill()
    attend(w, masks)


@pytest.mark.parametrize("n,new,per_kv", [(256, 1, 3), (257, 1, 3), (256, 70, 2), (260, 66, 2)])
def test_attention_of_the_most_sequences_that_are_cut(n, new, per_kv):
    """256 sequences, the longest of them cut, and more, which are whole."""
    past = [(37 * i) % 50 + (700 if i % 64 == 5 else 0) for i in range(n)]
    w = World(past, [1 + (i * new) // n for i in range(n)], seed=n + new, kv_heads=1, per_kv=per_kv)
    w.fill()
    a = attend(w)
    assert torch.equal(a, attend(w))


@pytest.mark.parametrize("past,new,per_kv", [([16500], 64, 4), ([9000, 70], 64, 4), ([16500], 8, 4), ([9000, 70, 3], 16, 2)])
def test_attention_of_drafts_over_long_contexts(past, new, per_kv):
    """Many pieces to be joined, of 32 rows and of 128, with a short sequence beside them."""
    w = World(past, [new] * len(past), seed=new + len(past), kv_heads=8, per_kv=per_kv, group=64, bf16=len(past) > 1)
    masks, _ = tree_masks(w.g, w.new)
    w.fill()
    a = attend(w, masks)
    out = torch.empty_like(a)
    w.cache.attend(w.batch(w.mask_tensor(masks)), w.q.cuda(), out, SCALE, None, stream())
    assert torch.equal(a, out)


def attend_with_loose_bounds(w, masks, tokens=1 << 22):
    """As attend, but the call's bound of tokens is far beyond the sequences, as in a captured step of a server: blocks of 128 rows are
    then chosen where they fit the rows."""
    table = torch.full((len(w.new), tokens // w.page_tokens), -1, dtype=torch.int32, device="cuda")
    table[:, : w.table.shape[1]] = w.table
    batch = kvc.CacheBatch(w.new_start, w.tokens, table, w.most_new, tokens, w.num_pages, None if masks is None else w.mask_tensor(masks))
    outs = []
    for _ in range(2):
        out = torch.full_like(w.q, float("nan"), device="cuda")
        stat = torch.full(w.q.shape[:2], float("nan"), device="cuda")
        w.cache.attend(batch, w.q.cuda(), out, SCALE, stat, stream())
        outs.append(out)
    assert not w.cache.status.any() and torch.equal(*outs)
    w.check_attention(out, stat, SCALE, masks)


@pytest.mark.parametrize("bits_k,bits_v,group", list(itertools.product((4, 8), (4, 8), (32, 64, 128))))
@pytest.mark.parametrize("bf16,transform", [(False, 0), (True, 0), (False, 1), (True, 1)])
def test_attention_of_every_kind_with_loose_bounds(bits_k, bits_v, group, bf16, transform):
    w = World([0, 900, 45], [37, 37, 1], seed=group, kv_heads=1, per_kv=6, bf16=bf16, bits_k=bits_k, bits_v=bits_v, group=group,
              transform=transform, block_tokens=32, limits={"tokens": 1 << 22})
    w.page_tokens = 32
    masks, _ = tree_masks(w.g, w.new)
    w.fill()
    attend_with_loose_bounds(w, masks)


@pytest.mark.parametrize("past,new,per_kv,trees", [([16500], 64, 4, True), ([9000, 70], 64, 4, True), ([300, 0, 7000], 100, 5, False),
                                                   ([4000], 16, 8, True), ([5000, 31], 1, 4, False), ([700], 8, 4, True)])
def test_long_contexts_with_loose_bounds(past, new, per_kv, trees):
    w = World(past, [new] * len(past), seed=new + len(past), kv_heads=4, per_kv=per_kv, group=64, bf16=len(past) > 1, block_tokens=64,
              limits={"tokens": 1 << 22})
    w.page_tokens = 64
    masks = tree_masks(w.g, w.new)[0] if trees else None
    w.fill()
    attend_with_loose_bounds(w, masks)


def test_rows_that_see_nothing():
    """Empty mask rows: zeros and -infinity where there is no context, the context alone where there is one; and rows that see later
    drafts, or not themselves."""
    w = World([0, 9, 0, 300], [6, 6, 1, 40], seed=4)
    masks = [[0, 1, 0, 0b111111, 0b100000, 0], [0, 0, 0b10, 0b100001, 0, 0b11], [0], [0] * 40]
    w.fill()
    out = attend(w, masks)
    assert (out[0] == 0).all() and (out[12] == 0).all()


def test_nan_rows_that_nobody_sees():
    """K and V rows of NaN and infinity in masked places do not reach rows that do not see them."""
    w = World([40], [8], seed=5)
    masks = [[0b1, 0b11, 0b101, 0b1001, 0b1, 0b1, 0b1, 0b1]]
    w.k[0][46] = w.v[0][46] = float("nan")
    w.k[0][47] = w.v[0][47] = float("inf")
    w.fill()
    attend(w, masks)


@pytest.mark.parametrize("scale", [0.0, -0.11, 3.0])
def test_scales_and_sharp_scores(scale):
    w = World([700], [3], seed=6, bits_k=8)
    w.fill()
    attend(w, scale=scale)


@pytest.mark.parametrize("bf16,size", [(False, 3000.0), (False, 1e-4), (True, 1e20), (True, 1e-30)])
def test_queries_of_any_size(bf16, size):
    w = World([200], [2], seed=7, bf16=bf16)
    w.q = (w.q.float() * size).to(w.dtype)
    w.q[1, 0] = 0.0
    w.q[0, 1, 3] = w.q[0, 1, 3] * 0.001
    w.fill()
    attend(w, scale=float(SCALE / size))


def test_values_at_the_types_limit():
    """Values whose top code stands for more than 65504, and tiny ones."""
    w = World([100], [1], seed=9, spread=False)
    w.v[0][:, 0] = torch.where(torch.rand(101, DIM, generator=w.g) < 0.5, 65504.0, -65504.0).to(w.dtype)
    w.v[0][:, 1] = (torch.randn(101, DIM, generator=w.g) * 1e-6).to(w.dtype)
    w.fill()
    out = torch.empty_like(w.q, device="cuda")
    w.cache.attend(w.batch(), w.q.cuda(), out, SCALE, None, stream())
    assert torch.isfinite(out).all()
    w.check_attention(out, None, SCALE)


def test_many_sequences_and_workspace():
    """Odd lengths, some sequences without new rows, several workgroups per sequence; twice the same bits."""
    g = torch.Generator().manual_seed(1)
    past = torch.randint(0, 900, (23,), generator=g).tolist()
    w = World(past, [0 if i % 5 == 3 else 1 for i in range(23)], seed=2, kv_heads=1, per_kv=2)
    w.fill()
    assert w.plan.workspace_size() > 0
    a = attend(w)
    assert torch.equal(a, attend(w))


def test_strided_queries_and_outputs():
    w = World([50, 3], [4, 9], seed=10, per_kv=3)
    w.fill()
    fused = torch.randn(13, 12, DIM, device="cuda").to(w.dtype)
    fused[:, 2:8] = w.q.cuda()
    out = torch.full((13, 9, DIM), 3.0, dtype=w.dtype, device="cuda")
    w.cache.attend(w.batch(), fused[:, 2:8], out[:, 1:7], SCALE, None, stream())
    w.check_attention(out[:, 1:7], None, SCALE)
    assert (out[:, [0, 7, 8]] == 3.0).all()


@pytest.mark.parametrize("bits_k,bits_v,group,block_tokens", [(4, 4, 32, 16), (8, 4, 64, 32), (4, 8, 128, 16), (8, 8, 32, 64)])
def test_accepted_drafts_move(bits_k, bits_v, group, block_tokens):
    w = World([14, 0, 31, 100, 5], [40, 33, 1, 64, 7], seed=11, kv_heads=5, bits_k=bits_k, bits_v=bits_v, group=group, block_tokens=block_tokens)
    w.fill()
    keep = [[0, 1, 5, 6, 17, 18, 19, 20, 21, 22, 23, 24, 25, 26, 27, 28, 29, 30, 39], list(range(33)), [0], [1, 63], []]
    start, flat = w.starts([len(k) for k in keep]), torch.tensor(sum(keep, []), dtype=torch.int32, device="cuda")
    w.cache.keep(w.batch(), start, flat, stream())
    expect = []
    for s, (p, n) in enumerate(zip(w.past, w.new)):
        at = list(range(p + n))
        for i, j in enumerate(keep[s]):
            at[p + i] = p + j
        expect.append(at)
    check_rows(w, expect)


def test_paths_of_trees():
    w = World([30, 64, 1], [21, 64, 9], seed=12)
    masks, paths = tree_masks(w.g, w.new)
    w.fill()
    attend(w, masks)
    w.cache.keep(w.batch(), w.starts([len(p) for p in paths]), torch.tensor(sum(paths, []), dtype=torch.int32, device="cuda"), stream())
    expect = [list(range(t)) for t in w.total]
    for s in range(3):
        for i, j in enumerate(paths[s]):
            expect[s][w.past[s] + i] = w.past[s] + j
    check_rows(w, expect)


def test_indices_that_do_not_fit():
    w = World([8, 8, 8, 8, 8], [6, 6, 6, 6, 6], seed=13)
    w.fill()
    before = w.cache.pages.clone()
    keep = [[2, 1], [0, 6], [-1], [3, 3], [2]]
    w.cache.keep(w.batch(), w.starts([len(k) for k in keep]), torch.tensor(sum(keep, []), dtype=torch.int32, device="cuda"), stream())
    assert w.cache.status.tolist() == [kvc.DEV_BAD_ROW] * 4 + [0]
    after = read_after = w.cache.pages
    assert not torch.equal(before, read_after)
    w.cache.status.zero_()
    expect = [list(range(14)) for _ in range(5)]
    expect[4][8] = 10
    check_rows(w, expect)
    # a start array that runs past the indices
    w.cache.keep(w.batch(), torch.tensor([0, 0, 0, 0, 0, 3], dtype=torch.int32, device="cuda"),
                 torch.tensor([0, 1], dtype=torch.int32, device="cuda"), stream())
    assert w.cache.status.tolist() == [0, 0, 0, 0, kvc.DEV_BAD_ROW]
    assert after.data_ptr() == w.cache.pages.data_ptr()


def test_pages_outside_the_pool():
    """Entries out of range: reported, not read or written; attention goes on with the other tokens."""
    w = World([70, 70], [2, 2], seed=14)
    w.fill()
    good = w.table.clone()
    w.table[0, 1], w.table[0, 2] = w.num_pages, -5
    before = w.cache.pages.clone()
    out = torch.full_like(w.q, 9.0, device="cuda")
    w.cache.attend(w.batch(), w.q.cuda(), out, SCALE, None, stream())
    assert w.cache.status.tolist() == [kvc.DEV_BAD_BLOCK, 0]
    w.cache.status.zero_()
    # the same as a sequence without those 32 tokens
    k, v, total = w.k[0], w.v[0], list(w.total)
    keep = list(range(16)) + list(range(48, 72))
    w.k[0], w.v[0], w.past, w.total = k[keep], v[keep], [38, 70], [40, 72]
    w.check_attention(out, None, SCALE)
    w.k[0], w.v[0], w.past, w.total = k, v, [70, 70], total
    ones = torch.ones(144, 2, DIM, dtype=w.dtype, device="cuda")
    w.cache.store(w.all_batch(), ones, ones, stream())
    assert w.cache.status.tolist() == [kvc.DEV_BAD_BLOCK, 0]
    lost = good[0, 1:3].long()
    size = w.plan.page_bytes()
    pages, was = w.cache.pages[: w.num_pages * size].reshape(-1, size), before[: w.num_pages * size].reshape(-1, size)
    assert torch.equal(pages[lost], was[lost])
    back = torch.full_like(ones, 4.0)
    w.cache.load(w.all_batch(), back, back.clone(), stream())
    assert (back[16:48] == 4.0).all() and (back[:16] == 1.0).all() and (back[48:] == 1.0).all()


def test_numbers_that_do_not_fit():
    """Starts, lengths and counts outside the call's bounds: the sequence is left out and reported, the others are done."""
    w = World([20, 20, 20, 20, 20, 20], [2, 2, 2, 2, 2, 2], seed=15)
    w.fill()
    pages = w.cache.pages.clone()
    q = w.q.cuda()
    good = torch.empty_like(q)
    w.cache.attend(w.batch(), q, good, SCALE, None, stream())
    w.tokens = torch.tensor([22, 23, -4, 1, 22, 22], dtype=torch.int32, device="cuda")      # 23 > max_tokens, 1 < its new rows
    w.new_start = torch.tensor([0, 2, 4, 6, 8, 1000, 10], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 9.0)
    w.cache.attend(w.batch(), q, out, SCALE, None, stream())
    want = [0, 32, 32, 32, 32, 32]
    assert w.cache.status.tolist() == want
    assert torch.equal(out[:2], good[:2]) and (out[2:] == 9.0).all()
    k = torch.full((12, 2, DIM), 9.0, dtype=w.dtype, device="cuda")
    w.cache.status.zero_()
    w.cache.load(w.batch(), k, k.clone(), stream())
    assert w.cache.status.tolist() == want and (k[2:] == 9.0).all() and not (k[:2] == 9.0).any()
    w.new_start = torch.tensor([3, 2, 4, 6, 8, 10, 12], dtype=torch.int32, device="cuda")
    w.tokens = torch.tensor([22, 23, 40, 1, 0, 22], dtype=torch.int32, device="cuda")
    w.cache.status.zero_()
    w.cache.store(w.batch(), k, k, stream())
    assert w.cache.status.tolist() == [32, 32, 32, 32, 32, 0]
    assert not torch.equal(pages, w.cache.pages)


def test_on_another_stream():
    w = World([500], [4], seed=16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q = w.q.cuda()
        w.fill()
        out = torch.empty_like(q)
        w.cache.attend(w.batch(), q, out, SCALE, None, side.cuda_stream)
    side.synchronize()
    w.check_attention(out, None, SCALE)


def test_a_captured_step_follows_the_lengths():
    """A decoding step (store, attend) in a graph: the lengths, tables and rows change between the replays, the launches do not."""
    w = World([0], [90], seed=17, per_kv=8)
    k, v, q = torch.empty(1, 2, DIM, dtype=w.dtype, device="cuda"), torch.empty(1, 2, DIM, dtype=w.dtype, device="cuda"), \
        torch.empty(1, 16, DIM, dtype=w.dtype, device="cuda")
    out = torch.empty_like(q)
    tokens, start = torch.ones(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    b = kvc.CacheBatch(start, tokens, w.table, 1, 90, w.num_pages)

    def run(st):
        w.cache.store(b, k, v, st)
        w.cache.attend(b, q, out, SCALE, None, st)

    k.zero_(), v.zero_(), q.zero_()
    run(stream())
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(side.cuda_stream)
    outs = []
    for i in range(90):
        k.copy_(w.k[0][i: i + 1])
        v.copy_(w.v[0][i: i + 1])
        q.copy_(w.q[i: i + 1])
        tokens.fill_(i + 1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        outs.append(out.clone())
        if i % 30 == 29:                                  # eager work between the replays
            run(stream())
            torch.cuda.synchronize()
            assert torch.equal(out, outs[-1])
    assert not w.cache.status.any()
    w.check_attention(torch.cat(outs), None, SCALE)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB, with the pages of a sequence at both of its ends."""
    w = World([60], [5], seed=18, kv_heads=8, block_tokens=16, bits_k=8, bits_v=8)
    size = w.plan.page_bytes()
    pages = (5 << 30) // size
    w.cache = kvc.Cache(w.plan, pages)
    w.num_pages = pages
    w.table[0, :5] = torch.tensor([0, pages - 1, pages // 2, pages - 2, (1 << 32) // size], dtype=torch.int32)
    w.fill()
    check_rows(w)
    attend(w)


def test_one_row_or_head_with_any_stride():
    """A dimension of one thing has a stride that is never used: one row cut out of odd rows, one head with an odd stride."""
    w = World([40], [1], seed=31, per_kv=4)
    w.fill()
    want = attend(w)
    wide = torch.zeros(2, 8 * DIM + 3, dtype=w.dtype, device="cuda")
    q = wide.as_strided((1, 8, DIM), (8 * DIM + 3, DIM, 1))
    q.copy_(w.q)
    out = torch.zeros_like(wide).as_strided((1, 8, DIM), (8 * DIM + 3, DIM, 1))
    assert q.stride(0) % 8 and out.stride(0) % 8
    w.cache.attend(w.batch(), q, out, SCALE, None, stream())
    assert torch.equal(out, want) and not w.cache.status.any()
    w = World([3], [9], seed=32, kv_heads=1)
    w.fill()
    k = torch.zeros(9, 1, DIM, dtype=w.dtype, device="cuda").as_strided((9, 1, DIM), (DIM, 5, 1))
    v = torch.zeros_like(k).as_strided((9, 1, DIM), (DIM, 1, 1))
    w.cache.load(w.batch(), k, v, stream())
    hk, hv = w.held(0)
    assert np.array_equal(k.double().cpu().numpy(), hk.read_back(False)[3:]) and np.array_equal(v.double().cpu().numpy(), hv.read_back(False)[3:])


def test_tensors_of_the_host_are_refused():
    """Addresses that the GPU cannot follow never reach a kernel."""
    w = World([40], [2], seed=33)
    w.fill()
    out, host = torch.empty_like(w.q, device="cuda"), torch.empty_like(w.q)
    rows = torch.zeros(2, 2, DIM, dtype=w.dtype, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)                        # noqa: E731
    for call in (lambda: w.cache.attend(w.batch(), host, out, SCALE), lambda: w.cache.attend(w.batch(), out, host, SCALE),
                 lambda: w.cache.attend(w.batch(), out, out.clone(), SCALE, torch.zeros(out.shape[:2])),
                 lambda: w.cache.store(w.batch(), rows, rows.cpu()), lambda: w.cache.load(w.batch(), rows.cpu(), rows),
                 lambda: w.cache.keep(w.batch(), i32(0, 1), i32(0).cuda()), lambda: w.cache.keep(w.batch(), i32(0, 1).cuda(), i32(0)),
                 lambda: w.cache.store(kvc.CacheBatch(i32(0, 2), i32(42), torch.zeros(1, 3, dtype=torch.int32), 2, 42, 3), rows, rows),
                 lambda: kvc.CacheBatch(i32(0, 2), i32(42).cuda(), torch.zeros(1, 3, dtype=torch.int32), 2, 42, 3),
                 lambda: kvc.Cache(w.plan, 3, "cuda", workspace=torch.zeros(1 << 26, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
    assert not w.cache.status.any()
