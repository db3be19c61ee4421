"""A pool refuses a call before anything of it changes: nothing here touches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S


def cache(d=128, k=0x10000, token_stride=None):
    """A cache whose arrays nobody reads."""
    c = S.PagedCache.__new__(S.PagedCache)
    row = token_stride or d
    c.c = S.CPagedCache(k, 0x20000000, 8 * row, 8 * row, row, 8 * row, 8 * row, row, None, 0, 0, 0, 16, 1, d, 8, S.KV_BF16, 0)
    c.address, c.n_pages, c.page_size, c.device, c._copyable = C.addressof(c.c), 16, 8, torch.device("cpu"), False
    return c


@pytest.mark.parametrize("bad", [dict(d=80), dict(k=0x10008), dict(token_stride=132), dict(token_stride=64)])
def test_caches_that_cannot_be_copied_are_refused_first(bad):
    p = S.PagePool(2, 4, 16, 8, device="cpu")
    for call in (p.update, p.compact):
        with pytest.raises(S.ShadowKVError):                         # not by what comes later: the tensors are not on a GPU
            call(caches=[cache(), cache(**bad)])
        with pytest.raises(ValueError):
            call(caches=[cache()])
        with pytest.raises(ValueError, match="4096"):
            call(caches=[cache()] * 4097)


@pytest.mark.parametrize("bad", [0.5, 1.5, float("nan"), float("inf"), -1, 2 ** 31])
def test_numbers_that_are_not_whole_are_refused(bad):
    p = S.PagePool(2, 4, 16, 8, device="cpu")
    with pytest.raises(ValueError, match="n_new"):
        p.update(n_new=bad)
    with pytest.raises(ValueError, match="max_moves"):
        p.compact(max_moves=bad)
