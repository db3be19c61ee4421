"""Refusals of the rotary and paged-cache entry points, and their host logic: nothing here touches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S

FAKE = 0x10000        # never dereferenced: validation fails first


def heads(**kw):
    base = dict(data=FAKE, seq_stride=0, token_stride=512, head_stride=128, n_seqs=1, n_tokens=6, n_heads=4, dtype=S.KV_BF16)
    base.update(kw)
    return S.CHeads(*(base[f] for f, _ in S.CHeads._fields_))


def rope(**kw):
    return S.Rope(**{**dict(head_dim=128), **kw}).c_struct()


def cache(**kw):
    base = dict(k=FAKE, v=FAKE, k_page_stride=4096, k_head_stride=2048, k_token_stride=128, v_page_stride=4096, v_head_stride=2048,
                v_token_stride=128, page_table=FAKE, table_stride=10, batch=3, pages_per_seq=10, n_pages=50, n_kv_heads=2, head_dim=128,
                page_size=16, kv_dtype=S.KV_BF16, reserved=0)
    base.update(kw)
    return S.CPagedCache(*(base[f] for f, _ in S.CPagedCache._fields_))


def ref(x):
    return None if x is None else C.byref(x)


def rotate(r, x, out, positions=None, offset=None):
    return S.lib().shadowkv_rotate(ref(r), ref(x), ref(out), positions, offset, 0, None)


@pytest.mark.parametrize("bad", [dict(head_dim=80), dict(rot_dim=12), dict(rot_dim=136), dict(rot_dim=-8), dict(layout=2), dict(scaling=5), dict(scaling=-1),
                                 dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(magnitude=-1.0), dict(magnitude=float("inf")),
                                 dict(scaling=S.ROPE_LINEAR, factor=0.0), dict(scaling=S.ROPE_NTK, factor=float("nan")),
                                 dict(scaling=S.ROPE_BANDS, factor=8.0, low=4.0, high=4.0, original_len=8192),
                                 dict(scaling=S.ROPE_BANDS, factor=8.0, low=1.0, high=4.0),
                                 dict(scaling=S.ROPE_YARN, factor=8.0, low=0.0, high=32.0, original_len=4096),
                                 dict(scaling=S.ROPE_YARN, factor=8.0, low=1.0, high=32.0, original_len=4096, theta=1.0)])
def test_rope_refusals(bad):
    r = rope(**bad)
    assert rotate(r, heads(), heads()) == S.EINVAL and S.last_error()
    assert S.lib().shadowkv_rope_frequencies(C.byref(r), FAKE) == S.EINVAL
    k = heads(n_heads=2, token_stride=256)
    assert S.lib().shadowkv_paged_append(ref(cache()), ref(r), ref(k), ref(k), None, None, None, FAKE, None, None) == S.EINVAL


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=FAKE + 8), dict(n_heads=0), dict(n_seqs=-1), dict(n_tokens=-1), dict(dtype=2), dict(dtype=-1),
                                 dict(token_stride=516), dict(head_stride=-128), dict(n_seqs=1 << 16, n_tokens=1 << 16), dict(n_heads=70000)])
def test_heads_refusals(bad):
    x = heads(**bad)
    assert rotate(rope(), x, heads()) == S.EINVAL and S.last_error()
    assert rotate(rope(), heads(), x) == S.EINVAL


def test_rotate_refusals():
    r, x = rope(), heads()
    assert rotate(None, x, x) == S.EINVAL and rotate(r, None, x) == S.EINVAL and rotate(r, x, None) == S.EINVAL
    assert rotate(r, x, heads(n_tokens=5)) == S.EINVAL and "size" in S.last_error()
    assert rotate(r, x, heads(data=2 * FAKE), FAKE, FAKE) == S.EINVAL and "exclude" in S.last_error()
    # written arrays that overlap themselves: heads closer than d, a broadcast dimension
    assert rotate(r, x, heads(data=2 * FAKE, head_stride=64)) == S.EINVAL and "overlap" in S.last_error()
    assert rotate(r, x, heads(data=2 * FAKE, token_stride=0)) == S.EINVAL
    assert rotate(r, x, heads(token_stride=1024)) == S.EINVAL and "laid out differently" in S.last_error()
    # nothing to do is no error, and no pointer is needed
    none = heads(data=None, n_tokens=0)
    assert rotate(r, none, none) == S.OK
    inv = rope()
    inv.inv_freq, inv.scaling, inv.factor = FAKE, S.ROPE_LINEAR, 2.0
    assert rotate(inv, x, x) == S.EINVAL and "PLAIN" in S.last_error()
    inv.scaling = S.ROPE_PLAIN
    assert S.lib().shadowkv_rope_frequencies(C.byref(inv), FAKE) == S.EINVAL


def test_refusals_at_the_ends_of_the_ranges():
    # a stride that overflows when it is turned into bytes, factors that are finite in 64 bits only, more tokens than a launch has threads for
    assert rotate(rope(), heads(token_stride=(1 << 62) + 512), heads(data=2 * FAKE)) == S.EINVAL
    assert rotate(rope(magnitude=1e39), heads(), heads(data=2 * FAKE)) == S.EINVAL and "magnitude" in S.last_error()
    assert attend(scale=1e39) == S.EINVAL and attend(scale=2.5e38) == S.EINVAL and "softmax_scale" in S.last_error()
    many = dict(n_tokens=(1 << 27) + 3)
    assert rotate(rope(), heads(**many), heads(data=2 * FAKE, **many)) == S.EINVAL and "2^27" in S.last_error()
    k = heads(n_heads=2, token_stride=256, **many)
    assert append(cache(batch=1), k=k) == S.EINVAL and "2^27" in S.last_error()


def test_frequencies():
    f = S.Rope(128, theta=1e4).frequencies()
    assert f.shape == (64,) and f[0] == 1.0 and abs(f[32].item() - 1e-2) < 1e-16
    assert torch.allclose(S.Rope(128, theta=1e4, scaling=S.ROPE_LINEAR, factor=4.0).frequencies(), f / 4, rtol=1e-15, atol=0)
    bands = S.Rope(128, theta=1e4, scaling=S.ROPE_BANDS, factor=8.0, low=1.0, high=4.0, original_len=8192).frequencies()
    turns = 8192 * f / (2 * torch.pi)
    assert torch.equal(bands[turns > 4], f[turns > 4]) and torch.allclose(bands[turns < 1], f[turns < 1] / 8, rtol=1e-15, atol=0)
    yarn = S.Rope(128, theta=1e4, scaling=S.ROPE_YARN, factor=8.0, low=1.0, high=32.0, original_len=4096).frequencies()
    assert yarn[0] == f[0] and abs(yarn[-1] / f[-1] * 8 - 1) < 1e-14 and (yarn <= f).all() and (yarn[1:] < yarn[:-1]).all()


def append(c=None, r=None, k=None, v=None, q=None, q_out=None, starts=None, lens=FAKE):
    k = heads(n_heads=2, token_stride=256) if k is None else k
    return S.lib().shadowkv_paged_append(ref(c or cache()), ref(r), ref(k), ref(v or k), ref(q), ref(q_out), starts, lens, None, None)


def attend(c=None, q=None, out=None, starts=None, lens=FAKE, scale=0.0, ws=FAKE, n=1 << 40):
    q = heads() if q is None else q
    return S.lib().shadowkv_paged_attention(ref(c or cache()), ref(q), ref(out or heads(data=2 * FAKE)), None, starts, lens, 1, scale, ws, n, None)


@pytest.mark.parametrize("bad", [dict(batch=0), dict(pages_per_seq=0), dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=80), dict(page_size=0),
                                 dict(page_size=24), dict(page_size=1 << 17), dict(pages_per_seq=1 << 27, table_stride=1 << 27), dict(kv_dtype=3), dict(reserved=1),
                                 dict(table_stride=9), dict(k=None), dict(v=None), dict(page_table=None), dict(k=FAKE + 8), dict(v=FAKE + 2),
                                 dict(k_page_stride=4100), dict(v_token_stride=-128), dict(k_head_stride=2052)])
def test_cache_refusals(bad):
    c = cache(**bad)
    assert append(c) == S.EINVAL and S.last_error()
    assert attend(c) == S.EINVAL and S.last_error()


def test_append_refusals():
    k, q = heads(n_heads=2, token_stride=256), heads()
    assert append(cache(k_token_stride=64)) == S.EINVAL and "overlap" in S.last_error()
    assert append(k=heads(n_heads=3)) == S.EINVAL and append(k=heads(n_heads=2, n_seqs=2, seq_stride=4096)) == S.EINVAL
    assert append(v=heads(n_heads=2, n_tokens=5)) == S.EINVAL
    assert append(k=heads(n_heads=2, dtype=S.KV_FP8_E5M2)) == S.EINVAL                     # FP8 keys into a bf16 cache
    assert append(r=rope(head_dim=64)) == S.EINVAL and "head_dim" in S.last_error()
    assert append(q=q, q_out=q) == S.EINVAL and append(r=rope(), q=q) == S.EINVAL
    assert append(r=rope(), q=q, q_out=heads(n_heads=8, token_stride=1024)) == S.EINVAL
    assert append(r=rope(), q=heads(dtype=1), q_out=heads(dtype=1)) == S.EINVAL
    assert append(lens=None) == S.EINVAL
    assert append(k=heads(n_heads=2, n_tokens=7)) == S.EINVAL and "divide" in S.last_error()
    none = heads(n_heads=2, n_tokens=0, data=None)
    assert append(k=none) == S.OK


def test_attention_refusals():
    assert attend(q=heads(n_heads=3)) == S.EINVAL
    assert attend(cache(n_kv_heads=1), q=heads(n_heads=65), out=heads(n_heads=65, token_stride=65 * 128)) == S.EINVAL and "group" in S.last_error()
    assert attend(q=heads(dtype=1)) == S.EINVAL and attend(out=heads(dtype=1)) == S.EINVAL
    assert attend(out=heads(n_tokens=5)) == S.EINVAL and attend(out=heads(head_stride=64)) == S.EINVAL
    assert attend(scale=-1.0) == S.EINVAL and attend(scale=float("nan")) == S.EINVAL
    assert attend(lens=None) == S.EINVAL and attend(q=heads(n_tokens=7), out=heads(n_tokens=7)) == S.EINVAL
    assert attend(ws=None) == S.EWORKSPACE and attend(ws=FAKE + 16) == S.EWORKSPACE
    c = cache()
    need = S.lib().shadowkv_paged_attention_workspace_bytes(C.byref(c), 4, 6)
    assert need > 0 and need % 256 == 0 and attend(n=need - 1) == S.EWORKSPACE and "too small" in S.last_error()
    none = heads(n_tokens=0, data=None)
    assert attend(q=none, out=none) == S.OK
    assert S.lib().shadowkv_paged_attention_workspace_bytes(C.byref(c), 5, 6) == 0
    bare = cache(k=None, v=None, page_table=None)           # sizes are asked for before there are any arrays
    assert S.lib().shadowkv_paged_attention_workspace_bytes(C.byref(bare), 4, 6) == need


def test_python_refuses_what_is_not_on_the_gpu_or_of_another_shape():
    x = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        S.rotate(S.Rope(128), x)
    with pytest.raises(ValueError):
        S.rotate(S.Rope(128), x.float())
    with pytest.raises(ValueError):
        S.PagedCache(torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.PagedCache(torch.zeros(4, 2, 16, 128), torch.zeros(4, 2, 16, 128), torch.zeros(1, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.dense_pages(torch.zeros(2, 2, 40, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 40, 64, dtype=torch.bfloat16), 16)
