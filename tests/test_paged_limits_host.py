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


def test_written_arrays_that_share_memory_with_what_is_read():
    """Begun inside the other array, in another type, in another order: refused.  Interleaved and neighbouring arrays are not (a missing
    workspace is what they are refused for)."""
    r, x = rope(), heads()                                    # six tokens of four heads of 128, 2 bytes each: 6144 bytes
    for out in (heads(data=FAKE + 16), heads(data=FAKE + 1024), heads(data=FAKE + 6144 - 16), heads(data=FAKE - 16), heads(data=FAKE - 6144 + 16),
                heads(dtype=S.KV_FP8_E5M2), heads(data=FAKE + 256, token_stride=1024), heads(token_stride=128, head_stride=768),
                heads(data=FAKE + 768, head_stride=1024, token_stride=4096)):
        assert rotate(r, x, out) == S.EINVAL and "share memory" in S.last_error(), S.last_error()
        assert rotate(r, out, x) == S.EINVAL and "share memory" in S.last_error()
        if out.dtype == S.KV_BF16:
            c = cache()
            assert append(c, r=r, q=x, q_out=out) == S.EINVAL and "share memory" in S.last_error()
            assert attend(c, q=x, out=out) == S.EINVAL and "share memory" in S.last_error()
    wide = heads(token_stride=1024, head_stride=256)          # every other head of eight
    for a, b in ((x, heads(data=FAKE + 6144)), (x, heads(data=FAKE - 6144)), (x, x), (wide, heads(data=FAKE + 256, token_stride=1024, head_stride=256)),
                 (heads(token_stride=1024), heads(data=FAKE + 1024, token_stride=1024)), (heads(seq_stride=8), heads(seq_stride=512)),
                 (heads(n_heads=1, head_stride=0), heads(n_heads=1, head_stride=128))):
        assert attend(cache(n_kv_heads=1), q=a, out=b, ws=None) == S.EWORKSPACE, S.last_error()
        assert attend(cache(n_kv_heads=1), q=b, out=a, ws=None) == S.EWORKSPACE, S.last_error()


def test_arrays_that_span_more_than_there_is():
    for big in (dict(token_stride=1 << 47), dict(head_stride=1 << 46), dict(n_seqs=1 << 12, seq_stride=1 << 40, n_tokens=1)):
        assert rotate(rope(), heads(**big), heads(data=2 * FAKE)) == S.EINVAL and "span" in S.last_error(), S.last_error()
        assert rotate(rope(), heads(data=2 * FAKE), heads(**big)) == S.EINVAL and "span" in S.last_error()


def test_more_new_tokens_than_a_cache_has_room_for():
    """2^30 is what a sequence holds; beyond it, rows of blocks leave 32 bits."""
    many = dict(n_tokens=(1 << 31) - 1)
    assert attend(cache(batch=1), q=heads(**many), out=heads(data=1 << 45, **many), ws=None) == S.EINVAL and "2^30" in S.last_error()
    most = dict(n_tokens=1 << 30)
    assert attend(cache(batch=1), q=heads(**most), out=heads(data=1 << 45, **most), ws=None) == S.EWORKSPACE
    assert S.lib().shadowkv_paged_attention_workspace_bytes(C.byref(cache(batch=1)), 4, (1 << 31) - 1) == 0
