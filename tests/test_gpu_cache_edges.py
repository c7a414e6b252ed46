"""GPU tests (run with -m gpu) of the quantised cache at the edges of what its calls accept."""
import numpy as np
import pytest
import torch

from cache_util import DIM, World
from paper_2605_13734_amd import kvc

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("new,per_kv,most", [(1, 4, 5000), (9, 4, 1 << 22), (70, 4, 1 << 22), (1, 4, 200)])
@pytest.mark.parametrize("bf16,transform,tree", [(False, 0, False), (False, 1, True), (True, 0, True)])
def test_a_pool_without_pages(new, per_kv, most, bf16, transform, tree):
    """Every entry of the tables is out of range: nothing is read or written, attention gives zeros and -infinity."""
    past = [4900 if most >= 5000 else 100, 0, 3]
    dtype = torch.bfloat16 if bf16 else torch.float16
    plan = kvc.CachePlan(kvc.BF16 if bf16 else kvc.F16, 2, 2 * per_kv, DIM, 4, 8, 64, 16, transform, max_batch=4, max_tokens=most, max_new=new)
    cache = kvc.Cache(plan, 0)
    cache.pages.fill_(0x5a)
    table = torch.zeros(4, (most + 15) // 16, dtype=torch.int32, device="cuda")
    mask = torch.full((3 * new, (new + 63) // 64), -1, dtype=torch.int64, device="cuda") if tree else None
    batch = kvc.CacheBatch(i32(0, new, 2 * new, 3 * new, 3 * new), i32(*[p + new for p in past], 7), table, new, most, 0, mask)
    want = [kvc.DEV_BAD_BLOCK] * 3 + [0]
    q = torch.randn(3 * new, 2 * per_kv, DIM, device="cuda").to(dtype)
    for _ in range(2):
        out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
        cache.attend(batch, q, out, 0.1, lse, stream())
        assert cache.status.tolist() == want and (out == 0).all() and (lse == -np.inf).all()
        cache.status.zero_()
    rows = torch.full((3 * new, 2, DIM), 3.0, dtype=dtype, device="cuda")
    cache.store(batch, rows, rows, stream())
    cache.load(batch, rows, rows.clone(), stream())
    assert cache.status.tolist() == want and (rows == 3.0).all()
    cache.status.zero_()
    cache.keep(batch, i32(0, 1, 2, 3, 3), i32(new - 1, new - 1, new - 1), stream())
    assert cache.status.tolist() == want and (cache.pages == 0x5a).all()


def rows_without_numbers(rows, dtype):
    """Rows with NaN, with one infinity, with both, and, for bf16, with numbers whose sums leave 32 bits; the others are normal."""
    x = torch.randn(rows, 2, DIM, generator=torch.Generator().manual_seed(rows))
    x[1, 0, 9] = float("nan")
    x[2] = float("nan")
    x[4, 1, 0], x[4, 0, 100] = float("inf"), float("-inf")
    x[5, 1, 3], x[5, 1, 4] = float("inf"), float("-inf")
    x[7, 0, 127], x[7, 0, 64], x[7, 1, 1] = float("-inf"), float("nan"), float("nan")
    x[9] = 65504.0
    if dtype == torch.bfloat16:
        x[10] = 3.0e38
        x[11, :, ::2], x[11, :, 1::2] = 3.0e38, -3.0e38
        x[12, :, :64], x[12, :, 64:] = 3.0e38, -3.2e38
    return x.to(dtype)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("bits_k,group,transform", [(4, 32, 1), (8, 64, 1), (4, 128, 1), (8, 32, 0)])
@pytest.mark.parametrize("past,new", [(0, 32), (3, 27)])
def test_rows_that_hold_no_numbers(bf16, bits_k, group, transform, past, new):
    """NaN counts as 0, also where the rotation makes it of two infinities, and what is beyond the range as its limit; whole granules and
    parts of them.  Attention reads such a token as it is held."""
    w = World([past], [new], seed=group, bf16=bf16, bits_k=bits_k, group=group, transform=transform, spread=False)
    w.k[0][past: past + 16] = rows_without_numbers(16, w.dtype)
    w.v[0][past: past + 16] = rows_without_numbers(16, w.dtype).flip(1)
    w.fill()
    k, v = (torch.empty(past + new, 2, DIM, dtype=w.dtype, device="cuda") for _ in range(2))
    w.cache.load(w.all_batch(), k, v, stream())
    held_k, held_v = w.held(0)
    assert np.array_equal(k.double().cpu().numpy(), held_k.read_back(bf16)) and np.array_equal(v.double().cpu().numpy(), held_v.read_back(bf16))
    assert (k[past + 2] == 0).all()
    q, out = w.q.cuda() * 2.0 ** -12, torch.empty_like(w.q, device="cuda")
    w.q = q.cpu()
    w.cache.attend(w.batch(), q, out, 0.1, None, stream())
    w.check_attention(out, None, 0.1)
    assert not w.cache.status.any()


@pytest.mark.parametrize("exponent,scale", [(-124, 2.9e38), (-124, -2.9e38), (-131, 2.9e38), (-124, 2.0e36), (-118, 3.0e34)])
@pytest.mark.parametrize("new,transform,bits_k", [(2, 0, 4), (2, 1, 8), (40, 0, 8), (40, 1, 4)])
def test_smallest_queries_and_largest_scales(exponent, scale, new, transform, bits_k):
    """Queries near the smallest numbers of bf16, some below its normal ones, with scales that bring their scores to a few units; scales
    whose product with log2(e) is beyond the largest number."""
    w = World([200], [new], seed=7, bf16=True, bits_k=bits_k, transform=transform, spread=False)
    w.q = (w.q.float() * 2.0 ** exponent).to(w.dtype)
    w.fill()
    out, lse = torch.empty_like(w.q, device="cuda"), torch.empty(w.q.shape[:2], device="cuda")
    w.cache.attend(w.batch(), w.q.cuda(), out, scale, lse, stream())
    assert w.q.abs().max() > 0 and not w.cache.status.any()
    w.check_attention(out, lse, scale)


@pytest.mark.parametrize("exponent", [118, 121, 124])
@pytest.mark.parametrize("new,transform,bits_k,group", [(2, 0, 4, 32), (2, 1, 8, 128), (40, 0, 8, 128), (40, 1, 4, 64), (3, 0, 4, 128)])
def test_largest_queries(exponent, new, transform, bits_k, group):
    """Queries up to 2^127 whose channels have one sign for the most part, so that the sums of their groups are large, too."""
    w = World([200], [new], seed=7, bf16=True, bits_k=bits_k, transform=transform, group=group, spread=False)
    w.q = ((w.q.float() + 2.0).clamp(-1.0, 7.0) * 2.0 ** (exponent - (7 if transform else 0))).to(w.dtype)
    w.fill()
    out, lse, scale = torch.empty_like(w.q, device="cuda"), torch.empty(w.q.shape[:2], device="cuda"), 0.1 * 2.0 ** -exponent
    w.cache.attend(w.batch(), w.q.cuda(), out, scale, lse, stream())
    assert torch.isfinite(w.q).all() and not w.cache.status.any()
    w.check_attention(out, lse, scale)


@pytest.mark.parametrize("bf16,new,transform,past", [(False, 1, 0, 40), (True, 9, 1, 40), (False, 40, 0, 40), (True, 40, 1, 40), (False, 1, 0, 3000),
                                                     (True, 70, 0, 3000)])
def test_queries_that_are_no_numbers(bf16, new, transform, past):
    """A query with NaN or an infinity gives NaN, as a result and as its lse, and no other row; one that sees nothing gives zeros and
    -infinity whatever it is."""
    w = World([past], [new], seed=11, bf16=bf16, transform=transform)
    w.fill()
    q = w.q.cuda()
    lost = torch.zeros(w.q.shape[:2], dtype=torch.bool)
    for r, h, value in ((0, 1, "nan"), (0, 4, "inf"), (new - 1, 6, "-inf"), (new // 2, 7, "nan")):
        q[r, h, (5 * r + h) % DIM] = float(value)
        lost[r, h] = True
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    w.cache.attend(w.batch(), q, out, 0.1, lse, stream())
    assert torch.isnan(out.cpu()[lost]).all() and torch.isnan(lse.cpu()[lost]).all()
    good, good_lse = torch.empty_like(q), torch.empty_like(lse)
    w.cache.attend(w.batch(), w.q.cuda(), good, 0.1, good_lse, stream())
    out, lse = torch.where(lost.cuda()[:, :, None], good, out), torch.where(lost.cuda(), good_lse, lse)
    w.check_attention(out, lse, 0.1)
    if new > 1:
        w = World([0], [new], seed=12, bf16=bf16, transform=transform)
        w.fill()
        masks = [[0] + [1 << i for i in range(1, new)]]
        q = w.q.cuda()
        q[0] = float("nan")
        w.cache.attend(w.batch(w.mask_tensor(masks)), q, out, 0.1, lse, stream())
        assert (out[0] == 0).all() and (lse[0] == -np.inf).all()
        w.q[0] = 0.0
        w.check_attention(out, lse, 0.1, masks)


@pytest.mark.parametrize("new,bf16", [(1, False), (1, True), (40, False), (40, True)])
def test_scores_beyond_32_bits(new, bf16):
    """No sum of weights can be made of infinite scores: NaN, and not a row that sees nothing."""
    w = World([200], [new], seed=13, bf16=bf16)
    w.fill()
    out, lse = torch.zeros_like(w.q, device="cuda"), torch.zeros(w.q.shape[:2], device="cuda")
    w.cache.attend(w.batch(), w.q.cuda(), out, 3.0e38, lse, stream())
    assert torch.isnan(out).all() and torch.isnan(lse).all() and not w.cache.status.any()
