"""shadowkv_paged_attention where logits rise behind a sequence's first keys and a value nearly fills fp32: finite in, finite out."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8, Cache, check_attention

pytestmark = pytest.mark.gpu

LN2 = math.log(2.0)      # as softmax_scale: a logit of x is x in powers of two


@pytest.mark.parametrize("rise", [3.0, 7.0, 7.9375, 9.0, 30.0])
@pytest.mark.parametrize("n,seqs,L", [(1, 16, 4096), (4, 16, 4096), (100, 4, 3001)])
def test_a_value_near_the_largest_number_under_a_rising_maximum(n, seqs, L, rise):
    """Every key has logit 0 but one far behind the first, which is `rise` (in powers of two) above them and has a value of 1.5 * 2^126.
    Its softmax weight is below one, so the sum of weighted values fits in fp32, and so does the quotient."""
    d, hkv, hq = 128, 2, 8
    cache = Cache([L] * seqs, hkv, d, BF, 64, seed=1)
    for i in range(seqs):
        k = torch.zeros(L, hkv, d, device="cuda")
        v = cache.vd[i].float()
        at = L - n - 137 - 53 * i
        k[at, :, 0] = rise
        v[at, :, 3] = 1.5 * 2.0 ** 126 * (-1) ** i
        k, v = k.to(BF), v.to(BF)
        cache.put(i, k, v)
        cache.kd[i], cache.vd[i] = k.double(), v.double()
    q = torch.randn(n * seqs, hq, d, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(BF)
    q[..., 0] = 1.0
    lse = torch.empty(q.shape[:2], device="cuda")
    out = S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts([n] * seqs), softmax_scale=LN2, lse=lse)
    assert torch.isfinite(out.float()).all()
    check_attention(cache, q, out, lse, [n] * seqs, scale=LN2)


@pytest.mark.parametrize("n", [2, 40])
def test_the_smallest_values_keep_their_bits(n):
    """Values of a few of bf16's smallest steps (2^-133), equal along the keys: the mean is the value itself, however weights are scaled."""
    d, L = 64, 700
    cache = Cache([L], 2, d, BF, 16, seed=3)
    row = (torch.arange(d, device="cuda") % 7 + 1).to(torch.int16).view(BF)      # 1 ... 7 steps
    v = row.expand(L, 2, d).contiguous()
    cache.put(0, cache.kd[0].to(BF), v)
    cache.vd[0] = v.double()
    q = torch.randn(n, 8, d, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(BF)
    out = S.paged_attention(cache.c, q, cache.kv_lens())
    # off by the weights' rounding (a 2^-8 of at most 7 steps), then by half a step of the result's
    assert ((out.double() - row.double()).abs() <= (0.5 + 7 * 2.0 ** -7) * 2.0 ** -133).all()


@pytest.mark.parametrize("scale", [8.2e-39, 1e-30])
@pytest.mark.parametrize("n", [1, 70])
def test_the_smallest_scales_give_means(n, scale):
    cache = Cache([300, 90], 2, 96, F8, 16, seed=5, k_gain=8.0)
    q = torch.randn(2 * n, 8, 96, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(BF)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts([n, n]), softmax_scale=scale, lse=lse)
    check_attention(cache, q, out, lse, [n, n], scale=scale)
