"""GPU tests (run with -m gpu): norms and rotations with numbers at the ends of what the calls take."""
import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, check_rotation, heads, own_type, stream, typed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [kvc.ROTARY_HALVES, kvc.ROTARY_PAIRS])
@pytest.mark.parametrize("rotary_dim", [128, 64])
@pytest.mark.parametrize("size,weight,amplitude", [(1e18, 1e30, 1.0), (1e10, 1e36, 1.0), (1.0, 1e37, 1.0), (3e37, 1e34, 1.0), (1e-14, 1e-30, 1.0), (1e-14, 1e-37, 1.0),
                                                   (1e-30, 1e-36, 1.0), (1e5, 3e36, 8.0), (1e-12, 1e-28, 1e-5)])
def test_weights_of_norms_are_as_large_as_their_type(size, weight, amplitude, layout, rotary_dim):
    """bf16: a normed head times its weight stays inside 32 bits, though the head's own numbers times the weight do not."""
    eps = 1e-38 if size < 1 else 1e-6
    plan = kvc.PromptPlan(kvc.BF16, 2, 4, layout=layout, rotary_dim=rotary_dim, amplitude=amplitude, eps=eps)
    q, k, _ = heads(9, 2, 2, True, 3)
    q, k = ((x.double() * size).bfloat16() for x in (q, k))
    g = torch.Generator().manual_seed(5)
    w = [(weight * (1 + 0.3 * torch.randn(DIM, generator=g, dtype=torch.float64))).bfloat16().to(DEVICE) for _ in "qk"]
    at = torch.randint(0, 100000, (9,), generator=g, dtype=torch.int32)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    kvc.Prompt(plan).rotate(q, k, at.to(DEVICE), q_out, k_out, *w, stream=stream())
    f = kvc.rotary_frequencies(rotary_dim)
    for got, x, y in ((q_out, q, w[0]), (k_out, k, w[1])):
        assert got.isfinite().all()
        check_rotation(got, x, y, at.numpy(), f, layout == kvc.ROTARY_PAIRS, amplitude, eps, True)
