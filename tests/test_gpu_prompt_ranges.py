"""GPU tests (run with -m gpu): the attention over prompts where sums are long, and scores and values large or small."""
import math

import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, half_step, i32, own_type, stream, typed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16,heads,rows", [(False, 1, 5000), (True, 1, 8192), (False, 32, 4096), (False, 64, 32768), (True, 1, 32768), (False, 1, 131072), (True, 1, 131072)])
def test_sums_of_many_equal_weights(bf16, heads, rows):
    """The first score is 0, all others are b, below it: the additions of the weights could all round the same way (the scores are some for which
    sums of one weight after the other in 32 bits do: 0.0001 off behind 32k tokens).  Row i: log(1 + i e^b), and 1 where all values are.

    The logarithm: roundings of an exponent of up to 32 and of the exponential itself (32 * 2^-24 * ln 2 + 2^-23), sums (20 roundings: 20 * 2^-24),
    together below 2^-17; its own roundings in 32 bits, of a number and of its base-2 value with the weights' bias: below 2^-20 of it.
    The result: half a step for the weights, half a step for itself, 2^-24 for each product of 32 tokens that is added."""
    dtype = typed(bf16)
    prompt = kvc.Prompt(kvc.PromptPlan(own_type(bf16), heads, heads))
    q, k = torch.zeros(1, 1, DIM, dtype=dtype, device=DEVICE), torch.zeros(rows, 1, DIM, dtype=dtype, device=DEVICE)
    q[:, :, 0] = 1.0
    v = torch.ones(1, 1, DIM, dtype=dtype, device=DEVICE).expand(rows, heads, DIM)
    out, lse = torch.empty(rows, heads, DIM, dtype=dtype, device=DEVICE), torch.empty(rows, heads, device=DEVICE)
    count = torch.arange(rows, dtype=torch.float64, device=DEVICE)
    for b in (-0.55029296875, -0.65576171875, -0.59375, -0.81640625, -0.07421875):
        k[1:, :, 0] = b
        b = k[-1, 0, 0].item()               # (as the type has it)
        out.fill_(77.0)
        prompt.attend(kvc.PromptBatch(i32(0, rows), rows), q.expand(rows, heads, DIM), k.expand(rows, heads, DIM), v, out, 1.0, lse, stream())
        want = torch.log1p(count * math.exp(b))
        off = (lse[:, 0].double() - want).abs()
        assert (off <= 2.0 ** -17 + want * 2.0 ** -20).all(), (b, off.max(), off.argmax())
        assert torch.equal(lse, lse[:, :1].expand(lse.shape)) and torch.equal(out, out[:, :1].expand(out.shape))
        error = (out[:, 0].double() - 1).abs().amax(1)
        assert (error <= 2.02 * half_step(bf16) + 2.0 ** -18 + count / 32 * 2.0 ** -24).all(), (b, error.max(), error.argmax())


# (KV heads, query heads per KV head, rows of the tensors) of calls with blocks of 64 rows, of 64 shared by two sets of waves, of 128 and 192
BLOCKS = {(64, 4): (32, 2, 700), (64, 8): (1, 2, 900), (128, 4): (48, 2, 2600), (192, 4): (32, 2, 10000)}


@pytest.mark.parametrize("block", BLOCKS)
@pytest.mark.parametrize("bf16,large,scale", [(False, 15, 2.0 ** -7), (False, 15, 2.0 ** -3), (False, 15, -2.0 ** -7), (True, 50, 2.0 ** -77), (True, 50, 2.0 ** -70),
                                              (True, 50, 1.0), (True, 50, 1e30), (True, 50, -2.0 ** -77)])
def test_scores_far_from_zero(block, bf16, large, scale):
    """Scores that 32 bits hold, with differences that they hold too, and far larger than the differences that an exponential can tell.

    Queries (2^large, 1 or 2^(large + 10)), keys (0, -2^large or 2^large, j): scores 0 or +-2^(2 large) and the steps of such numbers, exactly.  Weights
    and the result are rounded to the type; 2^-17 allows for factors of up to 32 with two roundings (64 * 2^-24 is less) and the sums."""
    kv, per, rows = BLOCKS[block]
    dtype, n = typed(bf16), 640
    plan = kvc.PromptPlan(own_type(bf16), kv, kv * per)
    assert plan.block_rows(1, rows, rows) == block
    g = torch.Generator().manual_seed(large)
    step = 2.0 ** (2 * large - 23)           # of numbers from 2^(2 large)
    q, k = torch.zeros(rows, 1, DIM, dtype=torch.float64), torch.zeros(rows, 1, DIM, dtype=torch.float64)
    q[:, 0, 0], q[:, 0, 1] = 2.0 ** large, 1.0 if not bf16 else 2.0 ** (large + 10)
    # a part near zero, one far below it, one far above it
    k[100:250, 0, 0], k[250:, 0, 0] = -(2.0 ** large), 2.0 ** large
    k[:, 0, 1] = torch.randint(0, 8, (rows,), generator=g) * step / q[0, 0, 1]
    v = torch.randn(rows, 1, DIM, generator=g)
    q, k, v = (x.to(dtype).to(DEVICE) for x in (q, k, v))
    out, lse = torch.full((rows, kv * per, DIM), 77.0, dtype=dtype, device=DEVICE), torch.full((rows, kv * per), 77.0, device=DEVICE)
    kvc.Prompt(plan).attend(kvc.PromptBatch(i32(0, n), rows), q.expand(rows, kv * per, DIM), k.expand(rows, kv, DIM), v.expand(rows, kv, DIM), out, scale,
                            lse, stream())
    scores = torch.where(torch.ones(n, n, device=DEVICE).tril() > 0, q[:n, 0].double() @ k[:n, 0].double().T, math.copysign(math.inf, -scale))
    top = scores.amax(1, keepdim=True) if scale > 0 else scores.amin(1, keepdim=True)
    weights = torch.exp((scores - top) * scale)
    total = weights.sum(1, keepdim=True)
    want, size = weights / total @ v[:n, 0].double(), weights / total @ v[:n, 0].double().abs()
    u = half_step(bf16) * 1.01
    assert ((out[:n, 0].double() - want).abs() <= want.abs() * u + size * (u + 2.0 ** -17) + n * 2.0 ** -33 * 6).all()
    assert torch.equal(out[:n], out[:n, :1].expand(n, kv * per, DIM)) and (out[n:] == 77).all()
    want = (top * scale + total.log())[:, 0]
    off, some = (lse[:n, 0].double() - want).abs(), want.abs() < 3e38        # (others are beyond the logarithm's type)
    assert (off[some] <= 2.0 ** -17 + want.abs()[some] * 2.0 ** -21).all() and some.any()


@pytest.mark.parametrize("heads,rows,block", [(1, 20000, (64, 8)), (8, 12000, (64, 4)), (64, 30000, (192, 4)), (1, 1 << 20, (192, 4))])
def test_sums_of_the_largest_values_behind_a_lower_maximum(heads, rows, block):
    """bf16: a first tile of score 0, then scores just too low to become the maximum that weights refer to (6.9 in base 2, so each weighs 2^6.9): sums
    of up to a million of the largest values stay inside 32 bits.  All values are equal: half a step for the weights, half a step for the result,
    2^-18 for the sums, 2^-24 for each product of 32 tokens."""
    plan = kvc.PromptPlan(kvc.BF16, heads, heads)
    assert plan.block_rows(1, rows, rows) == block
    q, k = torch.zeros(1, 1, DIM, dtype=torch.bfloat16, device=DEVICE), torch.zeros(rows, 1, DIM, dtype=torch.bfloat16, device=DEVICE)
    q[:, :, 0] = 1.0
    k[64:, :, 0] = 4.78
    out = torch.empty(rows, heads, DIM, dtype=torch.bfloat16, device=DEVICE)
    allowed = 2.02 * half_step(True) + 2.0 ** -18 + torch.arange(rows, device=DEVICE) / 32 * 2.0 ** -24
    for value in (3.38e38, -3.38e38):
        v = torch.full((1, 1, DIM), value, dtype=torch.bfloat16, device=DEVICE)
        out.fill_(77.0)
        kvc.Prompt(plan).attend(kvc.PromptBatch(i32(0, rows), rows), *(x.expand(rows, heads, DIM) for x in (q, k, v)), out, 1.0, None, stream())
        got = out[:, 0].double() / v[0, 0, 0].double()
        assert ((got - 1).abs().amax(1) <= allowed).all(), (value, (got - 1).abs().amax())
        assert torch.equal(out, out[:, :1].expand(out.shape))


@pytest.mark.parametrize("block", BLOCKS)
@pytest.mark.parametrize("bf16", [False, True])
def test_means_of_the_largest_value_are_numbers(block, bf16):
    """A mean is no more than the largest value, also where weights that are rounded up would take it beyond the type; an infinite value stays one.  Half
    a step for the weights, half a step for the result, 2^-18 for the sums and 2^-24 for each product of 32 tokens."""
    kv, per, rows = BLOCKS[block]
    dtype, n = typed(bf16), 500
    plan = kvc.PromptPlan(own_type(bf16), kv, kv * per)
    assert plan.block_rows(1, rows, rows) == block
    q, k = torch.zeros(1, 1, DIM, dtype=dtype, device=DEVICE), torch.zeros(rows, 1, DIM, dtype=dtype, device=DEVICE)
    q[:, :, 0] = 1.0
    top = torch.finfo(dtype).max
    v = torch.full((rows, 1, DIM), top, dtype=dtype, device=DEVICE)
    v[:, :, ::2] = -top
    v[300, 0, 5], v[310, 0, 6] = math.inf, -math.inf
    out = torch.empty(rows, kv * per, DIM, dtype=dtype, device=DEVICE)
    allowed = 2.02 * half_step(bf16) + 2.0 ** -18 + n / 32 * 2.0 ** -24
    for i in range(1, 40):
        k[1:, :, 0] = -i / 16
        kvc.Prompt(plan).attend(kvc.PromptBatch(i32(0, n), rows), q.expand(rows, kv * per, DIM), k.expand(rows, kv, DIM), v.expand(rows, kv, DIM), out, 1.0,
                                None, stream())
        bits = out[:n].view(torch.int16)     # (some are no numbers)
        assert torch.equal(bits, bits[:, :1].expand(n, kv * per, DIM))
        got = out[:n, 0].double() / v[0, 0].double()
        assert not got[300:, 5].isfinite().any() and not got[310:, 6].isfinite().any()
        got[300:, 5] = got[310:, 6] = 1.0
        assert ((got - 1).abs() <= allowed).all(), (i, (got - 1).abs().max())
