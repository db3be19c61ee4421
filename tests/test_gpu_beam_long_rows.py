"""Rows of so many tokens that the sum of their exponentials meets the end of fp64's range."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.29, 1.34, 1.35, 1.4])
def test_millions_of_tokens_a_step_above_a_reference(scale):
    """Around 2^32 fp32 has steps of 512, which is 2^953 to 2^1034 at these scales.  Rows whose waves, nine chunks each, begin with a chunk a step below
    their largest logits: were those 2^998 (scale 1.35) each and counted relative to it, 2^26 of them would leave fp64's range."""
    period, n = 9 * 1024, 7282                                       # 65538 chunks: nine of a wave
    row = torch.full((n, period), 2.0 ** 32 + 512.0, device="cuda")
    row[:, :1024] = 2.0 ** 32
    got = S.beam_select(row.view(1, 1, -1), torch.zeros(1, 1, device="cuda"), n_out=4, logit_scale=scale)
    # equally likely but for 2^-953 of it: one rounding to fp32, and 2^-38 as everywhere
    want = -math.log(n * (period - 1024))
    assert got["tokens"][0].tolist() == [1024, 1025, 1026, 1027]
    assert ((got["scores"][0].double() - want).abs() <= 2.0 ** -24 * abs(want) + 2.0 ** -38).all()
