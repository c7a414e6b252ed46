"""GPU tests (run with -m gpu): the attention over prompts in each of the sizes of blocks that it is built in.  The sizes go by a call's
bounds, so the cases have many heads, which all hold the same numbers, and rows behind the sequences, until the size is the one that is
tested."""
import math

import numpy as np
import pytest
import torch

from paper_2605_13734_amd import kvc
from prompt_util import DEVICE, DIM, check_attention, i32, own_type, stream, typed

pytestmark = pytest.mark.gpu
SCALE = DIM ** -0.5
# (rows of a workgroup, waves): (KV heads, query heads per KV head, rows of the tensors)
KERNELS = {(64, 4): (32, 2, 700), (64, 8): (1, 2, 900), (128, 4): (48, 2, 2600), (192, 4): (32, 2, 10000)}


class Case:
    def __init__(self, kernel, lengths, bf16, seed, before=0):
        self.bf16 = bf16
        self.kv, self.per, self.rows = KERNELS[kernel]
        self.starts = (before + np.concatenate([[0], np.cumsum(lengths)])).tolist()
        assert self.starts[-1] <= self.rows
        self.prompt = kvc.Prompt(kvc.PromptPlan(own_type(bf16), self.kv, self.kv * self.per, max_batch=len(lengths)))
        self.most = self.rows                 # (a bound: the longest of all)
        assert self.prompt.plan.block_rows(len(lengths), self.most, self.rows) == kernel
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(3, self.rows, 1, DIM, generator=g)
        x[1] *= torch.exp(0.5 * torch.randn(DIM, generator=g))
        self.x = x.to(typed(bf16)).to(DEVICE)
        self.q, self.k, self.v = (y.expand(self.rows, n, DIM) for y, n in zip(self.x, (self.kv * self.per, self.kv, self.kv)))
        self.out = torch.full((self.rows, self.kv * self.per, DIM), 77.0, dtype=typed(bf16), device=DEVICE)
        self.lse = torch.full(self.out.shape[:2], 77.0, device=DEVICE)

    def run(self, scale=SCALE):
        self.prompt.attend(kvc.PromptBatch(i32(*self.starts), self.most), self.q, self.k, self.v, self.out, scale, self.lse, stream())
        assert not self.prompt.status.any()
        return self

    def check(self, scale=SCALE):
        q, k, v = self.x
        for a, b in zip(self.starts, self.starts[1:]):
            if b > a:
                check_attention(self.out[a:b, :1], self.lse[a:b, :1], q[a:b], k[a:b], v[a:b], scale, self.bf16)
        for x in (self.out, self.lse):
            assert torch.equal(x, x[:, :1].expand(x.shape))
            assert (x[: self.starts[0]] == 77).all() and (x[self.starts[-1]:] == 77).all()
        return self


LENGTHS = [[1, 2, 31, 32, 33, 0, 63, 64, 65, 95, 96, 97], [127, 128, 129, 191], [192, 193, 15], [255, 256, 100], [600], [448, 0, 17]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kernel", KERNELS)
def test_lengths(kernel, bf16, lengths):
    Case(kernel, lengths, bf16, sum(lengths), before=11).run().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kernel", KERNELS)
def test_all_rows(kernel, bf16):
    rows = KERNELS[kernel][2]
    Case(kernel, [rows], bf16, 1).run().check()
    Case(kernel, [rows - 33, 33], bf16, 2).run(-0.3).check(-0.3)


@pytest.mark.parametrize("kernel", KERNELS)
def test_rising_and_falling_scores(kernel):
    """Maxima that grow from tile to tile, and scores far below the first one, which the second set of waves has not seen."""
    for rising in (1, -1):
        c = Case(kernel, [640], False, 3)
        t = torch.linspace(0.2, 3.0, 640, device=DEVICE)
        c.x[0] = 1.0
        c.x[1, :640] = ((t if rising > 0 else t.flip(0))[:, None, None] * 10).half()
        c.run().check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("at", [0, 31, 32, 63, 64, 100, 191, 192, 349])
def test_what_is_not_seen_does_not_matter(kernel, bf16, at):
    clean = Case(kernel, [150, 350], bf16, at).run().check()
    for what, bad in ((1, math.nan), (2, math.nan), (2, -math.inf)):
        c = Case(kernel, [150, 350], bf16, at)
        c.x[what, 150 + at, 0, 40] = bad
        c.x[:, 500:] = bad                   # rows of no sequence
        c.run()
        same = torch.ones(c.out.shape, dtype=torch.bool, device=DEVICE)
        if what == 1:
            same[150 + at: 500] = False
            assert c.out[150 + at: 500].isnan().all() and c.lse[150 + at: 500].isnan().all()
            assert torch.equal(c.lse[: 150 + at], clean.lse[: 150 + at])
        else:
            same[150 + at: 500, :, 40] = False
            assert not c.out[150 + at: 500, :, 40].isfinite().any()
            assert torch.equal(c.lse, clean.lse)
        assert torch.equal(c.out[same], clean.out[same])


@pytest.mark.parametrize("kernel", KERNELS)
def test_minus_infinite_scores_weigh_nothing(kernel):
    """A first part of the tokens whose scores are -infinity: some tiles leave a row nothing."""
    c = Case(kernel, [400], True, 5)
    c.x[0] = c.x[0].abs() + 0.1
    c.x[1, :130] = -math.inf
    c.x[2, :130] = 9.0
    c.run()
    assert c.out[:130].isnan().all()
    alone = Case(kernel, [270], True, 5)
    alone.x[:, :270] = c.x[:, 130:400]
    alone.run()
    # (the same tokens, in other tiles: as far apart as two roundings of the weights and of the result)
    assert ((c.out[130:400].double() - alone.out[:270].double()).abs() <= 2.0 ** -6 * c.x[2, 130:400].abs().max()).all()
    assert (c.lse[130:400] - alone.lse[:270]).abs().max() < 1e-4


@pytest.mark.parametrize("kernel", KERNELS)
def test_equal_bits(kernel):
    c = Case(kernel, [333, 200], True, 6).run()
    first = c.out.clone(), c.lse.clone()
    for _ in range(5):
        c.out.fill_(77.0)
        c.run()
        assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])
