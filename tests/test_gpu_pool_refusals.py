"""Calls that a pool refuses leave it, and the caches, as they were."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import PlainPool, check_pool, moves_of

pytestmark = pytest.mark.gpu


def test_a_cache_that_cannot_be_copied_changes_nothing():
    pool, plain = S.PagePool(3, 5, 20, 4), PlainPool(3, 5, 20, 4)
    rand = lambda d: torch.randn(20, 2, 4, d, device="cuda").to(torch.bfloat16)  # noqa: E731
    good, bad = pool.cache(rand(64), rand(64)), [pool.cache(rand(80), rand(80)), pool.cache(rand(72)[..., 4:68], rand(64))]
    pool.update(n_new=6, caches=good)
    plain.update(None, None, 6)
    parents = torch.zeros(3, dtype=torch.int32, device="cuda")
    before = good.k.clone(), good.v.clone()
    for c in bad:
        with pytest.raises(S.ShadowKVError):
            pool.update(parents=parents, n_new=1, caches=[good, c])
        with pytest.raises(S.ShadowKVError):
            pool.compact(caches=[good, c])
    torch.cuda.synchronize()
    check_pool(pool, plain)
    assert torch.equal(good.k, before[0]) and torch.equal(good.v, before[1])
    pool.update(parents=parents, n_new=1, caches=good)               # and the call that is allowed forks them once
    moves, _ = plain.update([0, 0, 0], None, 1)
    check_pool(pool, plain)
    assert moves_of(pool) == moves
