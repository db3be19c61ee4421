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
