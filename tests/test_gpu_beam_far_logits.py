"""Sums over logits that lie far from zero and from each other, where a wave takes several chunks of 1024 tokens of a row one after the other: it does
so in calls of more than 8192 chunks.  Groups share their logits (a stride of 0), so that the same rows are summed a chunk at a time in a call of
one group, and two, four or all at a time in larger calls."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import LOGIT_TYPES, check_choice, choose

pytestmark = pytest.mark.gpu
CHUNK, VOCAB = 1024, 8 * 1024 - 37
GROUPS = [1, 512, 1024, 4096]                                        # of four rows of eight chunks: 1, 2, 4 and 8 chunks of a wave


def chunks(*values, vocab=VOCAB):
    """A row whose i-th chunk holds values[i] (the last one: all further chunks too)."""
    return torch.cat([torch.full((CHUNK,), float(v)) for v in values] + [torch.full((vocab,), float(values[-1]))])[:vocab]


def agrees(rows, groups, n, scale=1.0, slack=None):
    """rows [4, vocab], every group's.  check_choice's bound is for logits up to 2^10 (in units of the scale); for larger ones the products with
    the scale and the sums with the reference are rounded to 2^-53 of them, a few times: 2^-50."""
    x, s = rows[None].cuda(), torch.tensor([[0.0, -0.5, -1.0, -1.5]], device="cuda")
    want = choose(x, s.cpu(), n, scale=scale)
    if slack is None:
        slack = 2.0 ** -50 * scale * float(x[x.abs() < 1e6].abs().max())
    got = S.beam_select(x.expand(groups, -1, -1), s.expand(groups, -1).contiguous(), n_out=n, logit_scale=scale)
    got["parents"] = got["parents"] - 4 * torch.arange(groups, device="cuda", dtype=torch.int32)[:, None]
    for k, v in got.items():
        assert torch.equal(v, v[:1].expand_as(v)), k                 # equal logits have equal sums
    check_choice({k: v[:1] for k, v in got.items()}, want, slack)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [4, 6])
@pytest.mark.parametrize("groups", GROUPS)
def test_far_sums_beside_low_ones(groups, n, dtype):
    """Chunks far below zero, the later ones nearer to it, beside chunks that are as low as logits summed as they are may be."""
    rows = torch.stack([chunks(-10000, -9700, -550), chunks(-10000, -9670, -380), chunks(-550, -550, -9990, -9670, -550, -9700, -9500, -540),
                        chunks(-380, -20000, -19680, -19360, -19040, -380, -30000, -29680)])
    agrees(rows.to(LOGIT_TYPES[dtype]), groups, n)
    agrees(rows.to(LOGIT_TYPES[dtype]) / 16, groups, n, scale=16.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [4, 6])
@pytest.mark.parametrize("groups", GROUPS)
def test_far_sums_beside_high_ones(groups, n, dtype):
    rows = torch.stack([chunks(600, 5000, 5330, 600), chunks(615, 900, 615, 640, -30, 640), chunks(-550, 900, 1230, 1560, -550),
                        chunks(5000, 600, 4670, 5330, 600, -9000, 5000, 600)])
    agrees(rows.to(LOGIT_TYPES[dtype]), groups, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("step", [150, 328, 336, 500, 700, 1000])
@pytest.mark.parametrize("groups", GROUPS)
def test_references_that_move(groups, step, dtype):
    """Chunks that rise by less and by more than moves a row's reference (2^480, steps of 333), all of them far from zero or some of them near;
    and the same downwards."""
    gen = torch.Generator().manual_seed(step)
    up = chunks(*(step * i for i in range(8))) + torch.randn(VOCAB, generator=gen)
    rows = torch.stack([up - 20000, up - 4 * step, up + 3000, up.flip(0) - 20000])
    agrees(rows.to(LOGIT_TYPES[dtype]), groups, 6)
    agrees(rows.to(LOGIT_TYPES[dtype]), groups, 4, scale=0.37)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("mask", [-1e4, -3e4, "lowest", -math.inf])
@pytest.mark.parametrize("groups", GROUPS)
def test_masks(groups, mask, dtype):
    """One token in a hundred masked, nine of ten, whole chunks, all but a few tokens."""
    gen = torch.Generator().manual_seed(3)
    low = torch.finfo(LOGIT_TYPES[dtype]).min if mask == "lowest" else mask
    rows = (torch.randn(4, VOCAB, generator=gen) * 3).to(LOGIT_TYPES[dtype])
    rows[2] -= 500
    rows[0, torch.rand(VOCAB, generator=gen) < 0.01] = low
    rows[1, torch.rand(VOCAB, generator=gen) < 0.9] = low
    rows[2, CHUNK:3 * CHUNK], rows[2, 5 * CHUNK - 9:5 * CHUNK + 700] = low, low
    rows[3, 3:7 * CHUNK + 1], rows[3, 7 * CHUNK + 20:] = low, low
    agrees(rows, groups, 6, slack=2.0 ** -50 * 3e4)
    agrees(rows, groups, 4, slack=2.0 ** -50 * 3e4)


@pytest.mark.parametrize("groups", [1, 64, 400])
def test_a_large_vocabulary_at_a_low_temperature(groups):
    """50 chunks a row: logits around -49 at a scale of 10, a chunk around -85, the next around -60."""
    gen = torch.Generator().manual_seed(6)
    rows = -49.0 + 0.1 * torch.randn(4, 50257, generator=gen)
    for i, at in enumerate((0, 4, 16, 48)):                          # the first of a wave's, whether it takes 1, 2, 4, 8 or 10
        rows[i, at * CHUNK:(at + 1) * CHUNK] -= 36.0
        rows[i, (at + 1) * CHUNK:(at + 2) * CHUNK] -= 11.0
    agrees(rows, groups, 8, scale=10.0)


@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("order", [(0, 1, 1, 1, 1, 1, 1, 2), (0, 1, 0, 2, 1, 1, 3, 3), (3, 1, 1, 0, 0, 2, 1, 4), (0, 1, 2, 3, 4, 5, 6, 7)])
def test_logits_with_steps_as_large_as_what_moves_a_reference(groups, order):
    """Around 2^32 fp32 has steps of 512, 2^953 at this scale, and a step need not move the reference: a chunk's sum is up to 2^963 where two steps
    above it a single logit counts for everything.  Its score is 0 but for what is lost: everything else is 2^-943 of it."""
    x = chunks(*(2.0 ** 32 + 512.0 * k for k in order))
    top = max(order)
    for last in (0, 5):                                              # the largest logit once, in the last chunk that has it
        row = torch.where(x == 2.0 ** 32 + 512.0 * top, x - 512.0, x)
        row[VOCAB - 1 - last if order[-1] == top else order.index(top) * CHUNK + 40 + last] = 2.0 ** 32 + 512.0 * top
        rows = torch.stack([row, row + 512.0, row, row - 1024.0])
        agrees(rows, groups, 4, scale=1.29, slack=0.0)               # (differences of the logits are exact, and no more than 2^10 where they count)
