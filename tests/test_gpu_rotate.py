"""GPU tests (run with -m gpu): queries and keys normed per head and rotated by their positions, against 64-bit values."""
import math

import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, check_rotation, frequencies_of, heads, i32, own_type, stream, typed

pytestmark = pytest.mark.gpu


def world(kv_heads=2, per_kv=3, bf16=False, rows=9, seed=0, fused=False, **kw):
    plan = kvc.PromptPlan(own_type(bf16), kv_heads, kv_heads * per_kv, **kw)
    q, k, _ = heads(rows, kv_heads, per_kv, bf16, seed, fused)
    g = torch.Generator().manual_seed(seed + 1)
    w = [(1 + 0.3 * torch.randn(DIM, generator=g)).to(typed(bf16)).to(DEVICE) for _ in "qk"]
    at = torch.randint(0, 100000, (rows,), generator=g, dtype=torch.int32)
    return kvc.Prompt(plan), q, k, w, at


def check(q_out, k_out, q, k, w, at, bf16, layout=kvc.ROTARY_HALVES, amplitude=1.0, eps=None, **kw):
    f = frequencies_of(kw) or []
    for got, x, weight in ((q_out, q, w[0]), (k_out, k, w[1])):
        check_rotation(got, x, weight, at.cpu().numpy(), f, layout == kvc.ROTARY_PAIRS, amplitude, eps, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("eps", [None, 1e-6])
@pytest.mark.parametrize("layout", [kvc.ROTARY_HALVES, kvc.ROTARY_PAIRS])
@pytest.mark.parametrize("rotary_dim", [128, 112, 96, 64, 48, 16, 0])
def test_kinds(bf16, eps, layout, rotary_dim):
    kw = dict(rotary_dim=rotary_dim, layout=layout, eps=eps, amplitude=1.25 if rotary_dim % 32 else 1.0)
    for kv_heads, per_kv, rows in ((2, 3, 9), (1, 1, 1), (5, 1, 3)):
        prompt, q, k, w, at = world(kv_heads, per_kv, bf16, rows, rotary_dim, fused=True, **kw)
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        prompt.rotate(q, k, at.to(DEVICE), q_out, k_out, *w, stream=stream())
        check(q_out, k_out, q, k, w, at, bf16, **kw)


@pytest.mark.parametrize("kv_heads,per_kv,rows", [(8, 8, 1), (8, 4, 33), (4, 16, 100), (1, 2, 8191), (1, 2, 8192), (2, 5, 8300), (64, 1, 5)])
def test_sizes(kv_heads, per_kv, rows):
    """Few rows, whose heads are divided, and many."""
    for bf16 in (False, True):
        prompt, q, k, w, at = world(kv_heads, per_kv, bf16, rows, 3, eps=1e-5)
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        prompt.rotate(q, k, at.to(DEVICE), q_out, k_out, *w, stream=stream())
        check(q_out, k_out, q, k, w, at, bf16, eps=1e-5)


@pytest.mark.parametrize("scaling", [kvc.SCALE_LINEAR, kvc.SCALE_BASE, kvc.SCALE_BANDS, kvc.SCALE_RAMP])
def test_far_positions(scaling):
    """Angles of positions up to the largest number, with scaled frequencies: 2^-31 of a turn, and what the frequencies' 64 bits leave."""
    f = kvc.rotary_frequencies(128, 5e5, scaling, 8.0, 1.0, 32.0, 8192)
    for bf16 in (False, True):
        prompt, q, k, w, _ = world(rows=8, bf16=bf16, frequencies=f, seed=scaling)
        at = torch.tensor([0, 1, 2 ** 20, 10 ** 6 + 1, 2 ** 24 + 1, 10 ** 8 + 7, 2 ** 30 + 3, 2 ** 31 - 1], dtype=torch.int32)
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        prompt.rotate(q, k, at.to(DEVICE), q_out, k_out, stream=stream())
        check(q_out, k_out, q, k, w, at, bf16, frequencies=f)


def test_frequencies_of_any_sign_and_size():
    f = [-1.0, 0.0, 2 * math.pi, -2 * math.pi, math.pi, 7.5, 1e-12, -1e-3]
    prompt, q, k, w, at = world(rows=40, rotary_dim=16, frequencies=f)
    at = at % 1000
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    prompt.rotate(q, k, at.to(DEVICE), q_out, k_out, stream=stream())
    check(q_out, k_out, q, k, w, at, False, rotary_dim=16, frequencies=f)


@pytest.mark.parametrize("layout", [kvc.ROTARY_HALVES, kvc.ROTARY_PAIRS])
@pytest.mark.parametrize("eps", [None, 1e-6])
def test_in_place_one_at_a_time_and_left_as_they_are(layout, eps):
    """In place as into other tensors; q or k alone; rows with a position below zero stay."""
    prompt, q, k, w, at = world(2, 4, True, 50, 5, layout=layout, eps=eps)
    at[[0, 7, 49]] = torch.tensor([-1, -2 ** 31, -5], dtype=torch.int32)
    at = at.to(DEVICE)
    q_out, k_out = torch.full_like(q, 77.0), torch.full_like(k, 77.0)
    prompt.rotate(q, k, at, q_out, k_out, *w, stream=stream())
    assert (q_out[at < 0] == 77).all() and (k_out[at < 0] == 77).all() and not (q_out[at >= 0] == 77).all(-1).any()
    q2, k2 = q.clone(), k.clone()
    prompt.rotate(q2, k2, at, q_weight=w[0], k_weight=w[1], stream=stream())
    assert torch.equal(q2[at >= 0], q_out[at >= 0]) and torch.equal(k2[at >= 0], k_out[at >= 0])
    assert torch.equal(q2[at < 0], q[at < 0]) and torch.equal(k2[at < 0], k[at < 0])
    alone = torch.full_like(q, 77.0)
    prompt.rotate(q, None, at, alone, q_weight=w[0], stream=stream())
    assert torch.equal(alone, q_out)
    alone = torch.full_like(k, 77.0)
    prompt.rotate(None, k, at, None, alone, k_weight=w[1], stream=stream())
    assert torch.equal(alone, k_out)
    prompt.rotate(None, None, None, stream=stream())


def test_norms_alone_leave_rows_too():
    """Without a rotation positions are optional; given, they still say which rows are left as they are."""
    prompt, q, k, w, _ = world(2, 2, False, 6, 5, rotary_dim=0, eps=1e-6)
    at, outs = i32(3, -1, 0, -7, 9, 1), []
    for positions in (None, at):
        outs.append((torch.full_like(q, 77.0), torch.full_like(k, 77.0)))
        prompt.rotate(q, k, positions, *outs[-1], *w, stream=stream())
    check(*outs[0], q, k, w, at, False, rotary_dim=0, eps=1e-6)
    for x, y in zip(*outs):
        assert torch.equal(x[at >= 0], y[at >= 0]) and (y[at < 0] == 77).all()


def test_layouts():
    """Heads before rows, in and out; nothing between the heads is written."""
    prompt, q, k, w, at = world(2, 2, False, 70, 6, eps=1e-6)
    at = at.to(DEVICE)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    prompt.rotate(q, k, at, q_out, k_out, *w, stream=stream())
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k)]
    wide = torch.full((8, 70, 2 * DIM), 77.0, dtype=q.dtype, device=DEVICE)
    to = wide[:, :, :DIM].transpose(0, 1)
    prompt.rotate(*turned, at, to[:, :4], to[:, 5:7], *w, stream=stream())
    assert torch.equal(to[:, :4], q_out) and torch.equal(to[:, 5:7], k_out)
    assert (wide[:, :, DIM:] == 77).all() and (wide[4] == 77).all() and (wide[7] == 77).all()


@pytest.mark.parametrize("size,eps", [(1e30, 1e-6), (3e38, 1e-6), (1e-30, 0.0), (1e-38, 0.0), (2e19, 1e-6), (1e-25, 1e-6), (1.0, 1e20)])
def test_norms_of_large_and_small_heads(size, eps):
    """bf16 heads whose squares leave 32 bits, beside ordinary ones."""
    prompt, q, k, w, at = world(3, 3, True, 11, 7, eps=eps)
    for x in (q, k):
        big = torch.rand(x.shape[:2], device=DEVICE) < 0.5
        x[big] = (x[big].float() / 8 * size).bfloat16()
        x[0, 0] = (torch.sign(x[0, 0].float()) * size).bfloat16()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    prompt.rotate(q, k, at.to(DEVICE), q_out, k_out, *w, stream=stream())
    check(q_out, k_out, q, k, w, at, True, eps=eps)


@pytest.mark.parametrize("layout", [kvc.ROTARY_HALVES, kvc.ROTARY_PAIRS])
def test_no_numbers_stay_where_they_are(layout):
    """NaN and infinities spoil their pair, and with norms their head."""
    for eps in (None, 1e-6):
        for rotary_dim in (128, 64):
            kw = dict(layout=layout, eps=eps, rotary_dim=rotary_dim)
            prompt, q, k, w, at = world(2, 2, False, 20, 8, **kw)
            at = at.to(DEVICE)
            outs = []
            for bad in (False, True):
                x = q.clone()
                if bad:
                    x[3, 1, 10], x[4, 2, 100] = math.nan, math.inf
                q_out, k_out = torch.empty_like(q), torch.empty_like(k)
                prompt.rotate(x, k, at, q_out, k_out, *w, stream=stream())
                outs.append((q_out, k_out))
            assert torch.equal(outs[0][1], outs[1][1])
            same = torch.ones(q.shape, dtype=torch.bool, device=DEVICE)
            if eps is not None:
                same[3, 1] = same[4, 2] = False
                assert outs[1][0][3, 1].isnan().all()
            else:
                other = {(kvc.ROTARY_HALVES, 128): (74, 36), (kvc.ROTARY_HALVES, 64): (42, 100), (kvc.ROTARY_PAIRS, 128): (11, 101),
                         (kvc.ROTARY_PAIRS, 64): (11, 100)}[layout, rotary_dim]
                same[3, 1, [10, other[0]]] = False
                same[4, 2, [100, other[1]]] = False
                assert not outs[1][0][3, 1, [10, other[0]]].isfinite().any() and not outs[1][0][4, 2, 100].isfinite()
            assert torch.equal(outs[0][0][same], outs[1][0][same])


def test_zeros_and_top_values():
    """Heads of zeros give zeros; fp16 numbers that a rotation makes larger than the type's become infinite."""
    prompt, q, k, w, at = world(1, 2, False, 6, 9, eps=1e-6)
    q[:], k[:] = 0, 0
    prompt.rotate(q, k, at.to(DEVICE), q_weight=w[0], k_weight=w[1], stream=stream())
    assert not q.any() and not k.any()
    plain = kvc.Prompt(kvc.PromptPlan(kvc.F16, 1, 2))
    q[:] = 65504.0
    at = i32(*[0, 1, 2, 3, 4, 5])
    plain.rotate(q, None, at, stream=stream())
    assert (q[0] == 65504).all() and q[1].isinf().any() and not q.isnan().any()


def test_offsets_beyond_32_bits():
    rows, stride = 23000, 100000
    x = torch.empty(rows, stride, dtype=torch.bfloat16, device=DEVICE)
    q, out = (x[:, i * DIM: (i + 1) * DIM].unflatten(1, (1, DIM)) for i in range(2))
    q.copy_(torch.randn(q.shape, generator=torch.Generator(device=DEVICE).manual_seed(3), device=DEVICE))
    prompt, at = kvc.Prompt(kvc.PromptPlan(kvc.BF16, 1, 1)), torch.arange(rows, dtype=torch.int32, device=DEVICE)
    prompt.rotate(q, None, at, out, stream=stream())
    some = torch.tensor([0, 1, 21474, 21475, 22999], device=DEVICE)
    check_rotation(out[some], q[some], None, some.cpu().numpy(), kvc.rotary_frequencies(128), False, 1.0, None, True)


def test_captured_and_replayed():
    prompt, q, k, w, at = world(2, 4, True, 40, 10, eps=1e-6)
    at = at.to(DEVICE)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    call = lambda: prompt.rotate(q, k, at, q_out, k_out, *w, stream=stream())              # noqa: E731
    call()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call()
    for seed in range(3):
        at.copy_(torch.from_numpy(np.random.default_rng(seed).integers(0, 1 << 20, 40).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        check(q_out, k_out, q, k, w, at, True, eps=1e-6)
