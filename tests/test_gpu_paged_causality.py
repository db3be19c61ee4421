"""shadowkv_paged_attention: what a token does not see leaves its result as it is, to the last bit."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8, Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("n,hq,hkv,d", [(4, 8, 2, 128), (8, 8, 2, 64), (100, 8, 2, 128), (60, 6, 2, 96)])
def test_later_keys_of_any_size_change_nothing(n, hq, hkv, d, dtype):
    """Keys from some place on made 20 times as large, and values with them: the tokens before it get the same bits, with other tokens of their
    block looking at logits far beyond theirs."""
    L = 400
    for seed in range(6):
        at = L - n + 1 + seed * (n - 1) // 6                         # the first place that changes, one of the new tokens'
        cache = Cache([L], hkv, d, dtype, 16, seed=seed)
        q = torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(50 + seed), device="cuda").to(BF)
        lse = torch.empty(2, n, hq, device="cuda")
        was = S.paged_attention(cache.c, q, cache.kv_lens(), lse=lse[0])
        k, v = cache.kd[0].clone(), cache.vd[0].clone()
        k[at:] *= 20
        v[at:] *= 20
        cache.put(0, k.to(dtype), v.to(dtype))
        now = S.paged_attention(cache.c, q, cache.kv_lens(), lse=lse[1])
        same = at - (L - n)                                          # tokens that do not see it
        assert torch.equal(now[:same], was[:same]) and torch.equal(lse[0, :same], lse[1, :same]), f"seed {seed}"
        assert not torch.equal(now[same:], was[same:])


@pytest.mark.parametrize("n,hq", [(8, 4), (60, 8)])
def test_a_token_does_not_depend_on_the_queries_beside_it(n, hq):
    """Other tokens' queries made 20 times as large: the same bits for those that stay."""
    d, hkv, L = 128, 2, 900
    cache = Cache([L], hkv, d, BF, 16, seed=7)
    q = torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").to(BF)
    was = S.paged_attention(cache.c, q, cache.kv_lens())
    for keep in (0, n // 2, n - 1):
        other = (q.float() * 20).to(BF)
        other[keep] = q[keep]
        assert torch.equal(S.paged_attention(cache.c, other, cache.kv_lens())[keep], was[keep])
