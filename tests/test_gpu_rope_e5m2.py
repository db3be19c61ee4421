"""Rounding of computed fp32 numbers to E5M2 storage: full mantissas, ties, the ends of the range."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1.0, 1.125, 0.375, 1.0 + 2.0 ** -23, 1.5 - 2.0 ** -23, 2.0 ** -16 * 1.75, 57344.0 / 3.0])
@pytest.mark.parametrize("layout", [S.ROPE_HALF, S.ROPE_INTERLEAVED])
def test_products_round_once_to_nearest_even(layout, m):
    """At position 0 a rotation multiplies by the magnitude: every finite bf16 number times m, rounded to fp32, then as torch's cast."""
    d = 128
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF)
    bits = torch.where(torch.isfinite(bits.float()), bits, torch.zeros((), dtype=BF)).view(512, 1, d).cuda()
    out = torch.empty(bits.shape, dtype=F8, device="cuda")
    S.rotate(S.Rope(d, layout=layout, magnitude=m), bits, out=out, positions=torch.zeros(512, dtype=torch.int32, device="cuda"))
    x = bits.float() * torch.tensor(m, dtype=torch.float32, device="cuda")
    want = x.to(F8)
    assert torch.equal(out.float(), want.float())
