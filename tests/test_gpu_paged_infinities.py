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


@pytest.mark.parametrize("n,L", [(1, 64), (4, 300), (40, 64), (40, 1000), (40, 61)])
@pytest.mark.parametrize("causal", [False, True])
def test_logits_of_minus_infinity_throughout(n, L, causal):
    """Such a token gets zeros and a log-sum of minus infinity, infinite values or not."""
    cache = Cache([L, L], 2, 128, BF, 16, seed=6)
    k = cache.kd[0].to(BF)
    k[..., 0] = -math.inf
    v = cache.vd[0].to(BF)
    v[3, :, 7] = math.inf
    v[L - n, :, 8] = math.nan
    cache.put(0, k, v)
    q = _q(2 * n, 8, 128)
    q[..., 0] = 1.0
    out, lse = _attend(cache, q, [n, n], causal=causal)
    assert (out[:n] == 0).all() and (lse[:n] == -math.inf).all()
    assert torch.isfinite(out[n:].float()).all() and torch.isfinite(lse[n:]).all()


@pytest.mark.parametrize("n", [1, 4, 40])
def test_an_infinite_value_is_not_lost_where_its_weight_is(n):
    """A key whose weight lies below fp32's range, and so do those of every fourth run of 32 keys with it: its infinite value does not come
    out as a finite one, wherever it stands."""
    L, d = 260, 64
    for at in (2, 40, 70, 100, 130, 250):
        cache = Cache([L], 1, d, BF, 16, seed=7)
        k = torch.zeros(L, 1, d, device="cuda")
        k[torch.arange(L, device="cuda") // 32 % 4 == at // 32 % 4, 0, 0] = -400.0
        v = cache.vd[0].to(BF)
        v[at, 0, 9] = math.inf
        cache.put(0, k.to(BF), v)
        q = torch.zeros(n, 4, d, dtype=BF, device="cuda")
        q[..., 0] = 1.0
        out, _ = _attend(cache, q, [n], softmax_scale=math.log(2.0), causal=False)
        assert not torch.isfinite(out[..., 9].float()).any(), f"key {at}"
        assert torch.isfinite(out[..., 10:].float()).all() and torch.isfinite(out[..., :9].float()).all(), f"key {at}"
