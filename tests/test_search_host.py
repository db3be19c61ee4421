"""Refusals of a search's entry points, and the plain pool that the GPU tests compare with: nothing here touches a GPU."""
import ctypes as C
import random

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import PlainPool

FAKE = 0x10000        # never dereferenced: validation fails first
FAR = 0x10000000      # fakes of outputs, apart from each other


def make(struct, base, kw):
    base = {**base, **kw}
    return struct(*(base[f] for f, _ in struct._fields_))


def logits(**kw):
    return make(S.CLogits, dict(data=FAKE, group_stride=4000, beam_stride=1000, n_groups=2, n_beams=4, vocab=1000, dtype=0), kw)


def select(x=None, scores=FAR, finished=None, lengths=None, penalty=0.0, scale=0.0, end=-1, n=4, out=(2 * FAR, 3 * FAR, 4 * FAR), ended=None, long=None,
           ws=5 * FAR, room=1 << 20):
    x = logits() if x is None else x
    return S.lib().shadowkv_beam_select(C.byref(x), scores, finished, lengths, penalty, scale, end, n, *out, ended, long, ws, room, None)


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=FAKE + 1), dict(n_groups=-1), dict(n_beams=0), dict(n_beams=65), dict(vocab=0),
                                 dict(vocab=(1 << 30) + 1), dict(dtype=3), dict(dtype=-1), dict(group_stride=-1), dict(beam_stride=1 << 62),
                                 dict(n_groups=1 << 19), dict(data=FAKE + 2, dtype=2)])
def test_logits_refusals(bad):
    assert select(logits(**bad)) == S.EINVAL and S.last_error()


def test_select_refusals():
    assert S.lib().shadowkv_beam_select(None, FAR, None, None, 0.0, 0.0, -1, 4, FAR, FAR, FAR, None, None, FAR, 1, None) == S.EINVAL
    for bad in (dict(n=0), dict(n=65), dict(scores=None), dict(out=(None, 3 * FAR, 4 * FAR)), dict(out=(2 * FAR, None, 4 * FAR)),
                dict(out=(2 * FAR, 3 * FAR, None)), dict(penalty=17.0), dict(penalty=float("nan")), dict(penalty=1.0), dict(long=6 * FAR),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e39), dict(scale=1e-39), dict(end=-2), dict(end=1000)):
        assert select(**bad) == S.EINVAL and S.last_error(), bad
    # outputs on inputs: only as the same array, and only where there are as many places as beams
    assert select(out=(FAR + 4, 3 * FAR, 4 * FAR)) == S.EINVAL and "shares" in S.last_error()
    assert select(n=5, out=(FAR, 3 * FAR, 4 * FAR)) == S.EINVAL and "shares" in S.last_error()
    assert select(out=(2 * FAR, FAR, 4 * FAR)) == S.EINVAL and select(out=(2 * FAR, 2 * FAR, 4 * FAR)) == S.EINVAL
    assert select(out=(FAKE, 3 * FAR, 4 * FAR)) == S.EINVAL and select(ws=FAR) == S.EINVAL
    assert select(ws=None) == S.EWORKSPACE and select(ws=5 * FAR + 16) == S.EWORKSPACE
    need = S.lib().shadowkv_beam_select_workspace_bytes(C.byref(logits()), 4)
    assert need > 0 and need % 256 == 0 and select(room=need - 1) == S.EWORKSPACE
    assert S.lib().shadowkv_beam_select_workspace_bytes(C.byref(logits(data=None)), 4) == need
    assert S.lib().shadowkv_beam_select_workspace_bytes(C.byref(logits()), 65) == 0
    assert select(logits(n_groups=0, data=None), scores=None, ws=None) == S.OK


def rows(**kw):
    return make(S.CRows, dict(data=FAR, row_stride=1024, outer_stride=256, inner=256, n_outer=4, reserved=0), kw)


def reorder(*arrays, parents=FAKE, n=8):
    return S.lib().shadowkv_reorder_rows((S.CRows * max(len(arrays), 1))(*arrays), len(arrays), parents, n, None)


@pytest.mark.parametrize("bad", [dict(data=None), dict(row_stride=-1), dict(row_stride=1 << 60), dict(outer_stride=-256), dict(inner=-1), dict(n_outer=-1),
                                 dict(reserved=1), dict(inner=(1 << 48) + 1), dict(row_stride=1023), dict(outer_stride=255), dict(row_stride=0),
                                 dict(row_stride=100, outer_stride=512), dict(data=FAKE - 100)])
def test_rows_refusals(bad):
    assert reorder(rows(**bad)) == S.EINVAL and S.last_error()


def test_reorder_refusals():
    assert reorder(rows(), parents=None) == S.EINVAL and reorder(rows(), n=-1) == S.EINVAL and reorder(rows(), n=2049) == S.EINVAL
    assert S.lib().shadowkv_reorder_rows(None, 1, FAKE, 8, None) == S.EINVAL and S.lib().shadowkv_reorder_rows(None, -1, FAKE, 8, None) == S.EINVAL
    assert reorder(rows(), rows()) == S.EINVAL and "share" in S.last_error()
    assert reorder(rows(inner=100), rows(data=FAR + 99, inner=50)) == S.EINVAL
    assert reorder(rows(), rows(data=FAR + 7 * 1024 + 1000)) == S.EINVAL
    # nothing to do is no error, and no pointer is needed
    assert reorder(parents=None) == S.OK and reorder(rows(data=None), n=0) == S.OK and reorder(rows(data=None, inner=0)) == S.OK
    assert reorder(rows(data=None, n_outer=0)) == S.OK


def pool(**kw):
    return make(S.CPagePool, dict(page_table=7 * FAR, table_stride=10, kv_lens=8 * FAR, page_refs=9 * FAR, batch=3, pages_per_seq=10, n_pages=50, page_size=16), kw)


def moves(**kw):
    return make(S.CPageMoves, dict(src=10 * FAR, dst=11 * FAR, rows=12 * FAR, count=13 * FAR, capacity=3, reserved=0), kw)


def update(p=None, m=None, grow=1, ws=FAKE, room=1 << 20):
    p, m = p or pool(), m or moves()
    return S.lib().shadowkv_pages_update(C.byref(p), None, None, None, grow, C.byref(m), ws, room, None)


def compact(p=None, m=None, most=5, ws=FAKE, room=1 << 20):
    p, m = p or pool(), m or moves()
    return S.lib().shadowkv_pages_compact(C.byref(p), most, C.byref(m), None, ws, room, None)


@pytest.mark.parametrize("bad", [dict(page_table=None), dict(kv_lens=None), dict(page_refs=None), dict(batch=0), dict(batch=4097), dict(pages_per_seq=0),
                                 dict(n_pages=0), dict(n_pages=(1 << 28) + 1), dict(page_size=0), dict(page_size=24), dict(page_size=1 << 17),
                                 dict(table_stride=9), dict(table_stride=1 << 41), dict(pages_per_seq=1 << 27, table_stride=1 << 27)])
def test_pool_refusals(bad):
    assert update(pool(**bad)) == S.EINVAL and S.last_error()
    assert compact(pool(**bad)) == S.EINVAL


def test_update_and_compact_refusals():
    for bad in (dict(src=None), dict(dst=None), dict(rows=None), dict(count=None), dict(capacity=2), dict(capacity=-1), dict(reserved=1)):
        assert update(m=moves(**bad)) == S.EINVAL and S.last_error(), bad
    for bad in (dict(src=None), dict(dst=None), dict(count=None), dict(capacity=-1), dict(reserved=1)):
        assert compact(m=moves(**bad)) == S.EINVAL and S.last_error(), bad
    assert update(grow=-1) == S.EINVAL and compact(most=-1) == S.EINVAL
    assert S.lib().shadowkv_pages_update(None, None, None, None, 0, C.byref(moves()), FAKE, 1 << 20, None) == S.EINVAL
    assert S.lib().shadowkv_pages_update(C.byref(pool()), None, None, None, 0, None, FAKE, 1 << 20, None) == S.EINVAL
    need = S.lib().shadowkv_pages_workspace_bytes(C.byref(pool(page_table=None)))
    assert need > 0 and need % 256 == 0
    for call in (update, compact):
        assert call(ws=None) == S.EWORKSPACE and call(ws=FAKE + 8) == S.EWORKSPACE and call(room=need - 1) == S.EWORKSPACE
    assert S.lib().shadowkv_pages_workspace_bytes(C.byref(pool(batch=0))) == 0
    # arguments that share memory
    for where in (7 * FAR, 8 * FAR + 8, 9 * FAR + 196, 10 * FAR, 13 * FAR - 4, FAKE):
        for place in range(3):
            args = [None] * 3
            args[place] = where
            p, m = pool(), moves()
            assert S.lib().shadowkv_pages_update(C.byref(p), *args, 0, C.byref(m), FAKE, 1 << 20, None) == S.EINVAL and "share" in S.last_error()
    for bad in (dict(src=11 * FAR), dict(rows=9 * FAR), dict(count=8 * FAR + 4), dict(dst=7 * FAR + 100)):
        assert update(m=moves(**bad)) == S.EINVAL and "share" in S.last_error()
        assert compact(m=moves(**bad)) == S.EINVAL and "share" in S.last_error()
    assert update(pool(kv_lens=9 * FAR)) == S.EINVAL and compact(pool(page_table=FAKE)) == S.EINVAL


def cache(**kw):
    return make(S.CPagedCache, dict(k=FAKE, v=FAKE, k_page_stride=4096, k_head_stride=2048, k_token_stride=128, v_page_stride=4096, v_head_stride=2048,
                                    v_token_stride=128, page_table=None, table_stride=0, batch=0, pages_per_seq=0, n_pages=50, n_kv_heads=2,
                                    head_dim=128, page_size=16, kv_dtype=S.KV_BF16, reserved=0), kw)


def copy(frm, to, m=None, n=None):
    ptrs = C.POINTER(S.CPagedCache) * max(len(frm), 1)
    f, t, m = ptrs(*(C.pointer(c) for c in frm)), ptrs(*(C.pointer(c) for c in to)), m or moves(count=None)
    return S.lib().shadowkv_pages_copy(f, t, len(frm) if n is None else n, C.byref(m), None)


def test_copy_refusals():
    a = cache()
    for bad in (dict(n_kv_heads=1), dict(head_dim=64), dict(page_size=8), dict(kv_dtype=1), dict(k=None), dict(v=FAKE + 8), dict(n_pages=0), dict(page_size=24),
                dict(head_dim=80), dict(k_token_stride=64), dict(v_head_stride=2052), dict(reserved=1)):
        assert copy([a], [cache(**bad)]) == S.EINVAL and S.last_error(), bad
    assert copy([a], [a], n=-1) == S.EINVAL and copy([a], [a], n=4097) == S.EINVAL
    assert S.lib().shadowkv_pages_copy(None, None, 1, C.byref(moves()), None) == S.EINVAL
    for bad in (dict(src=None), dict(dst=None), dict(capacity=-1), dict(reserved=1)):
        assert copy([a], [a], moves(**bad)) == S.EINVAL, bad
    assert copy([], []) == S.OK and copy([a], [a], moves(src=None, dst=None, capacity=0)) == S.OK


def test_python_refuses_what_is_not_on_the_gpu_or_of_another_shape():
    with pytest.raises(ValueError):
        S.beam_select(torch.zeros(2, 3, 10), torch.zeros(2, 3))
    with pytest.raises(ValueError):
        S.reorder_rows(torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        S.pages_copy([], torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(S.ShadowKVError):
        S.PagePool(0, 4, 16, 16, device="cpu")
    with pytest.raises(ValueError):
        S.PagePool(2 ** 32 + 2, 4, 16, 16, device="cpu")
    p = S.PagePool(2, 4, 16, 16, device="cpu")
    for call in (p.update, p.compact):
        with pytest.raises(ValueError):
            call()
    for bad in (-1, 2 ** 32):
        with pytest.raises(ValueError):
            p.update(n_new=bad)
        with pytest.raises(ValueError):
            p.compact(max_moves=bad)
    with pytest.raises(ValueError):
        p.update(n_new=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        p.cache(torch.zeros(16, 1, 8, 64, dtype=torch.bfloat16), torch.zeros(16, 1, 8, 64, dtype=torch.bfloat16))


def test_the_plain_pool_keeps_its_own_rules():
    """What rows hold is counted, free pages are held by nobody, and rows share only what they have in common."""
    rng = random.Random(3)
    for _ in range(60):
        ps, batch, width = rng.choice([1, 4, 16]), rng.randint(1, 6), rng.randint(1, 6)
        p = PlainPool(batch, width, rng.randint(1, 30), ps)
        text = [[] for _ in range(batch)]                    # what each row's tokens are, written page by page
        store, serial = {}, 0
        for _ in range(12):
            parents = [rng.randint(-1, batch) for _ in range(batch)] if rng.random() < 0.6 else None
            keep = [rng.randint(-1, width * ps) for _ in range(batch)] if rng.random() < 0.4 else None
            n_new = [rng.randint(-1, 2 * ps) for _ in range(batch)]
            moves, kept = p.update(parents, keep, n_new)
            old = text
            text = [list(old[parents[i] if parents else i][:kept[i]]) if kept[i] else [] for i in range(batch)]
            for src, dst, n in moves:
                for j in range(n):
                    store[dst, j] = store[src, j]
            for i in range(batch):
                for at in range(kept[i], p.lens[i]):
                    serial += 1
                    text[i].append(serial)
                    store[p.rows[i][at // ps], at % ps] = serial
            if rng.random() < 0.3:
                done, used = p.compact(rng.choice([0, 1, 100]))
                for src, dst in done:
                    for j in range(ps):
                        if (src, j) in store:
                            store[dst, j] = store[src, j]
                assert not any(p.refs[used:])
            counts = [0] * p.n_pages
            for i in range(batch):
                assert len(p.rows[i]) == -(-p.lens[i] // ps) and len(text[i]) == p.lens[i]
                for page in p.rows[i]:
                    counts[page] += 1
                assert [store[p.rows[i][at // ps], at % ps] for at in range(p.lens[i])] == text[i]
            assert counts == p.refs
