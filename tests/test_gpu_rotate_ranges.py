"""GPU tests (run with -m gpu): norms and rotations with numbers at the ends of what the calls take."""
import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, check_rotation, half_step, heads, smallest, stream

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


def turns(position, frequency):
    """The part of a turn of an angle, from whole numbers: 1 / (2 pi) to 600 bits by pi = 16 arctan(1/5) - 4 arctan(1/239)."""
    bits = 700

    def arctan_of_one_by(x):
        term, total, n, sign = (1 << bits) // x, 0, 1, 1
        while term:
            total, term, n, sign = total + sign * (term // n), term // (x * x), n + 2, -sign
        return total
    two_pi = 8 * (4 * arctan_of_one_by(5) - arctan_of_one_by(239))
    top, bottom = frequency.as_integer_ratio()
    part = (position * top << 2 * bits) // (bottom * two_pi) & ((1 << bits) - 1)
    return (part >> (bits - 64)) / 2.0 ** 64


@pytest.mark.parametrize("layout", [kvc.ROTARY_HALVES, kvc.ROTARY_PAIRS])
def test_frequencies_of_many_turns_at_far_positions(layout):
    """Frequencies up to the largest that a plan takes: the whole turns are dropped without a bit of what is left (a quotient of 64 bits is off by 2^-7
    of a turn at the last of these).  2^-19 of the terms stands for 32-bit cosines (2^-21) and products; then the type's half step."""
    f = [1e9, -1e9, 123456789.125, -87654321.1, 1e7, 1e6 + 0.1, 2.0 ** 29, 999999999.9999]
    at = [2 ** 31 - 1, 2 ** 31 - 2, 10 ** 9 + 7, 2 ** 30 + 3, 10 ** 8 + 7, 123457, 1, 0]
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, 2, 6, layout=layout, rotary_dim=16, frequencies=f))
    q, k, _ = heads(len(at), 2, 3, False, 4)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    prompt.rotate(q, k, torch.tensor(at, dtype=torch.int32, device=DEVICE), q_out, k_out, stream=stream())
    angle = 2 * np.pi * np.array([[turns(p, x) for x in f] for p in at])
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    first, second = (slice(0, 16, 2), slice(1, 16, 2)) if layout == kvc.ROTARY_PAIRS else (slice(0, 8), slice(8, 16))
    for x, got in ((q, q_out), (k, k_out)):
        x, got = x.double().cpu().numpy(), got.double().cpu().numpy()
        a, b = x[..., first], x[..., second]
        for want, there in ((a * c - b * s, first), (a * s + b * c, second)):
            assert (np.abs(got[..., there] - want) <= np.abs(want) * half_step(False) * 1.01 + (np.abs(a) + np.abs(b)) * 2.0 ** -19 + smallest(False)).all()
        assert (got[..., 16:] == x[..., 16:]).all()


@pytest.mark.parametrize("rows,parts", [((1 << 26) + 1027, "q"), ((1 << 25) + 1, "qk")])
def test_more_rows_than_a_launch_has(rows, parts):
    """Rows that need more threads than one launch may have (17 GB): as calls of a quarter of them."""
    plan = kvc.PromptPlan(kvc.F16, 1, 1, rotary_dim=32)
    prompt, some = kvc.Prompt(plan), 4099
    block = torch.randn(some, 1, DIM, generator=torch.Generator().manual_seed(3)).half().to(DEVICE)
    at = torch.arange(rows, dtype=torch.int32, device=DEVICE)
    at[-5:-3] = -1                           # (left as they are)
    whole = []
    for _ in parts:
        x = torch.empty(rows, 1, DIM, dtype=torch.float16, device=DEVICE)
        for a in range(0, rows, some):
            x[a: a + some] = block[: rows - a]
        whole.append(x)
    q, k = whole[0], whole[1] if parts == "qk" else None
    prompt.rotate(q, k, at, stream=stream())
    piece = rows // 4 + 7
    for a in range(0, rows, piece):
        n = min(piece, rows - a)
        want = block[torch.arange(a, a + n, device=DEVICE) % some]
        prompt.rotate(want, None, at[a: a + n], stream=stream())
        for x in whole:
            assert torch.equal(x[a: a + n], want)
