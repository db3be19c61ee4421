"""In-place and neighbouring views of one array through the rotary and paged-cache entry points."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, Cache, check_turned

pytestmark = pytest.mark.gpu


def _x(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


def test_in_place_through_two_views_of_one_token():
    """[b, h, 1, d] seen as [b, 1, h, d] by transposing and by viewing: the strides of the dimension of one differ, the memory does not."""
    r = S.Rope(128)
    a = _x(1, 5, 4, 1, 128)
    was = a.clone().view(5, 1, 4, 128)
    x, out = a.transpose(1, 2), a.view(5, 1, 4, 128)
    assert x.stride() != out.stride()
    off = torch.arange(100, 105, dtype=torch.int32, device="cuda")
    assert S.rotate(r, x, out=out, pos_offset=off) is out
    check_turned(r, out, was, off[:, None])


def test_heads_of_one_projection_beside_each_other():
    """q, k and v of one array, q rotated into every other head of another, and out of attention beside its q."""
    t, hq, hkv, d = 40, 8, 2, 64
    qkv = _x(2, t, hq + 2 * hkv, d)
    cache = Cache([0], hkv, d, BF, 16, spare=3, width=3)
    cache.table_cpu = torch.arange(3, dtype=torch.int32)[None]
    c = S.PagedCache(cache.k, cache.v, cache.table_cpu.cuda())
    lens = torch.tensor([t], dtype=torch.int32, device="cuda")
    both = torch.zeros(t, 2 * hq, d, dtype=BF, device="cuda")
    r = S.Rope(d)
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    want = S.paged_append(c, k, v, lens, rope=r, q=q)
    S.paged_append(c, k, v, lens, rope=r, q=q, q_out=both[:, ::2])
    assert torch.equal(both[:, ::2], want) and (both[:, 1::2] == 0).all()
    S.paged_attention(c, both[:, ::2], lens, out=both[:, 1::2])
    assert torch.equal(both[:, 1::2], S.paged_attention(c, want, lens)) and torch.equal(both[:, ::2], want)
    with pytest.raises(S.ShadowKVError, match="share memory"):
        S.paged_append(c, k[:-1], v[:-1], lens, rope=r, q=q[:-1], q_out=q[1:])


def test_starts_that_reach_beyond_the_rows():
    """Held to the rows there are, for appending as for attention: the last row goes to the last place."""
    t, hkv, hq, d = 9, 2, 4, 64
    cache = Cache([20, 33], hkv, d, BF, 16, seed=3)
    k, v, q = _x(1, t, hkv, d), _x(2, t, hkv, d), _x(3, t, hq, d)
    r, lens = S.Rope(d), cache.kv_lens()
    got = []
    for starts in ([0, 4, t], [-3, 4, t + 5]):
        c = S.PagedCache(cache.k.clone(), cache.v.clone(), cache.table)
        starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        qq = S.paged_append(c, k, v, lens, seq_starts=starts, rope=r, q=q)
        got.append((c.k.view(torch.int16), c.v.view(torch.int16), qq, S.paged_attention(c, qq, lens, seq_starts=starts)))
    for a, b in zip(*got):
        assert torch.equal(a, b)
