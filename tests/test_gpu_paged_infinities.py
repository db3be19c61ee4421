"""shadowkv_paged_attention with infinities that a token does see: in any tile, with any number of rows."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8, Cache

pytestmark = pytest.mark.gpu


def _attend(cache, q, news, **kw):
    lse = torch.full(q.shape[:2], 123.0, device="cuda")
    out = S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts(news), lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


def _q(n, hq, d, seed=1):
    return torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
@pytest.mark.parametrize("n,d,hq", [(1, 128, 2), (1, 96, 8), (4, 64, 8), (4, 128, 14), (100, 128, 8)])
def test_an_infinite_value_in_a_tile_that_all_rows_see(n, d, hq, bad, equal, dtype):
    """Keys 5 and 70 of 300, seen by every token: their element is infinite for each of them, every other one as without.  equal: all
    logits are the same, so that the weights are whole powers of two before they are normalised."""
    L, hkv = 300, 2
    cache = Cache([L], hkv, d, dtype, 16, seed=5)
    if equal:
        cache.put(0, torch.zeros(L, hkv, d, device="cuda").to(dtype), cache.vd[0].to(dtype))
    q = _q(n, hq, d)
    clean, clean_lse = _attend(cache, q, [n])
    for at, e in ((5, 5), (70, d - 1)):
        cache.v[int(cache.table_cpu[0, at // 16]), 1, at % 16, e] = bad
    out, lse = _attend(cache, q, [n])
    assert torch.equal(out[:, :hq // 2], clean[:, :hq // 2]) and torch.equal(lse, clean_lse)
    for e in (5, d - 1):
        assert (out[:, hq // 2:, e].float() == bad).all()
    rest = [e for e in range(d) if e not in (5, d - 1)]
    assert torch.equal(out[:, hq // 2:, rest], clean[:, hq // 2:, rest])
