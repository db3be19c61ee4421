"""Refusals of the rotary and paged-cache entry points at the ends of what they take; nothing here touches a GPU."""
import ctypes as C

from paper_2410_21465_amd import shadowkv as S
from test_paged_host import FAKE, append, attend, cache, heads, ref, rope, rotate


def test_softmax_scales_that_vanish_in_fp32():
    """Times log2(e) the scale has to be a normal fp32 number: 2^-126 = 1.1755e-38."""
    for scale in (1e-46, 5e-324, 1e-40, 8e-39):
        assert attend(scale=scale) == S.EINVAL and "softmax_scale" in S.last_error()
    for scale in (0.0, 8.2e-39, 1e-30):
        assert attend(scale=scale, ws=None) == S.EWORKSPACE          # (accepted: the workspace is looked at next)


def test_arrays_that_span_more_than_there_is():
    for big in (dict(token_stride=1 << 47), dict(head_stride=1 << 46), dict(n_seqs=1 << 12, seq_stride=1 << 40, n_tokens=1)):
        assert rotate(rope(), heads(**big), heads(data=2 * FAKE)) == S.EINVAL and "span" in S.last_error(), S.last_error()
        assert rotate(rope(), heads(data=2 * FAKE), heads(**big)) == S.EINVAL and "span" in S.last_error()
