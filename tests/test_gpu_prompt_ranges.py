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
