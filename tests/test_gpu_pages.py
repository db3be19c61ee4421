"""Pages that are forked, freed, grown, compacted and copied, against a pool that handles one row after the other."""
import random

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import PlainPool, check_pool, moves_of, put_pool

pytestmark = pytest.mark.gpu
BF, F8 = torch.bfloat16, torch.float8_e5m2


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def step(pool, plain, parents=None, keep=None, n_new=0, **kw):
    pool.update(parents=ints(parents), keep_lens=ints(keep), n_new=n_new if isinstance(n_new, int) else ints(n_new), **kw)
    moves, _ = plain.update(parents, keep, n_new)
    check_pool(pool, plain)
    assert moves_of(pool) == moves
    return moves


@pytest.mark.parametrize("batch,width,n_pages,ps", [(1, 1, 1, 1), (1, 5, 3, 16), (4, 9, 20, 4), (7, 3, 100, 64), (33, 40, 400, 8), (64, 20, 200, 2), (130, 6, 1000, 16),
                                                    (300, 700, 20000, 16), (1025, 4, 5000, 8), (4096, 3, 9000, 4)])
def test_random_walks(batch, width, n_pages, ps):
    rng = random.Random(batch * 7 + width)
    pool, plain = S.PagePool(batch, width, n_pages, ps), PlainPool(batch, width, n_pages, ps)
    check_pool(pool, plain)
    for turn in range(12):
        parents = None
        if rng.random() < 0.7:
            parents = [i if rng.random() < 0.5 else rng.randint(-1, batch) for i in range(batch)]
        keep = [rng.randint(-1, width * ps + 3) for _ in range(batch)] if rng.random() < 0.4 else None
        n_new = rng.choice([0, 1, ps, rng.randint(0, 3 * ps)]) if rng.random() < 0.5 else [
            rng.choice([0, 1, 1, -3, rng.randint(0, 2 * ps), rng.randint(0, width * ps)]) for _ in range(batch)]
        step(pool, plain, parents, keep, n_new)
        if turn % 4 == 3:
            most = rng.choice([0, 1, 5, None])
            used = pool.compact(max_moves=most)
            moves, end = plain.compact(1 << 30 if most is None else most)
            check_pool(pool, plain)
            assert [m[:2] for m in moves_of(pool)] == moves and int(used) == end
            assert all(m[2] == ps for m in moves_of(pool))


def test_holders_outside_the_table():
    """A prefix kept for later: its pages are not written, not given out, and moved with everything else."""
    pool, plain = S.PagePool(3, 8, 12, 4), PlainPool(3, 8, 12, 4)
    step(pool, plain, n_new=[6, 0, 0])
    plain.refs[1] += 1                                               # the partly filled second page
    plain.refs[7] += 1
    put_pool(pool, plain)
    assert step(pool, plain, [0, 0, 0], None, 1) == [(1, 2, 2), (1, 3, 2), (1, 4, 2)]
    step(pool, plain, [-1, -1, -1])
    assert plain.refs == [0, 1] + [0] * 5 + [1] + [0] * 4
    pool.compact()
    plain.compact(100)
    check_pool(pool, plain)


def test_pages_that_do_not_suffice():
    pool, plain = S.PagePool(5, 8, 9, 4), PlainPool(5, 8, 9, 4)
    step(pool, plain, n_new=[6, 4, 0, 3, 0])                         # 2 + 1 + 1 pages
    step(pool, plain, [0, 0, 0, 3, 1], None, [1, 9, 9, 1, 30])       # copies and pages of some, and of nobody behind them
    assert plain.lens[0] == 7 and plain.lens[3] == 4 and plain.lens[4] == 4
    step(pool, plain, None, [0, 0, 7, 4, 4], [0, 0, 1, 0, 32])
    step(pool, plain, None, None, [0, 0, 0, 0, 33])
    step(pool, plain, [-1] * 5, None, 100)                           # more than a row's table has entries
    assert plain.refs == [0] * 9


def test_entries_that_are_no_pages():
    pool, plain = S.PagePool(3, 6, 10, 4), PlainPool(3, 6, 10, 4)
    step(pool, plain, n_new=[10, 3, 5])
    for bad in (-1, 10, 2 ** 31 - 1, -2 ** 31):
        plain.rows[0][1] = plain.rows[0][2] = bad
        plain.rows[2][1] = bad
        plain.refs = [sum(p == q for r in plain.rows for q in r) for p in range(10)]
        put_pool(pool, plain)
        step(pool, plain, [0, 0, 2], None, 1)
        pool.compact()
        plain.compact(100)
        check_pool(pool, plain)


def test_parents_and_lengths_outside_their_ranges():
    pool, plain = S.PagePool(4, 5, 30, 4), PlainPool(4, 5, 30, 4)
    step(pool, plain, n_new=[20, 7, 1, 0])
    step(pool, plain, [2 ** 31 - 1, 1, -2 ** 31, 1], [2 ** 31 - 1, -2 ** 31, 9, 6], [2 ** 31 - 1, -5, 21, 14])
    pool.kv_lens.copy_(ints([2 ** 31 - 1, -7, 0, 0]))                # lengths that a row cannot have are held to what it can
    pool.update(n_new=0)
    assert pool.kv_lens.tolist() == [20, 0, 0, 0]


def contents(cache, table, lens, ps):
    """Tokens of every row, [n, h, d] of keys and values."""
    out = []
    for i, n in enumerate(lens):
        pages = table[i, :-(-n // ps)].long()
        out.append([x.view(torch.uint8 if x.element_size() == 1 else torch.int16)[pages].transpose(1, 2).flatten(0, 1)[:n] for x in (cache.k, cache.v)])
    return out


def page_arrays(n_pages, h, ps, d, dtype, layout, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = {"pages": (n_pages, h, ps, d), "tokens": (n_pages, ps, h, d), "heads": (h, n_pages, ps, d), "padded": (n_pages + 1, h + 1, ps, 2 * d)}[layout]
    perm = {"tokens": (0, 2, 1, 3), "heads": (1, 0, 2, 3)}.get(layout, (0, 1, 2, 3))
    x = torch.randn(shape, generator=gen, device="cuda").to(dtype).permute(perm)
    return x[1:, 1:, :, :d] if layout == "padded" else x


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("layout", ["pages", "tokens", "heads", "padded"])
@pytest.mark.parametrize("h,ps,d", [(2, 16, 128), (3, 4, 64), (1, 64, 96), (5, 1, 64)])
def test_rows_keep_what_they_hold(dtype, layout, h, ps, d):
    """Contents of every row through forks, cuts, growth and compaction, in three layers."""
    rng = random.Random(h * ps + d)
    batch, width, n_pages = 6, 9, 60
    pool, plain = S.PagePool(batch, width, n_pages, ps), PlainPool(batch, width, n_pages, ps)
    caches = [pool.cache(*(page_arrays(n_pages, h, ps, d, dtype, layout, 10 * l + i) for i in range(2))) for l in range(3)]
    for turn in range(8):
        before = [contents(c, pool.page_table, plain.lens, ps) for c in caches]
        parents = [rng.randint(-1 if turn else 0, batch - 1) for _ in range(batch)]
        keep = [rng.randint(0, width * ps) for _ in range(batch)] if turn % 3 == 2 else None
        n_new = [rng.randint(0, 2 * ps) for _ in range(batch)]
        _, kept = PlainPool.update(plain, parents, keep, n_new)
        pool.update(ints(parents), ints(keep), ints(n_new), caches=caches)
        check_pool(pool, plain)
        if turn % 3 == 1:
            pool.compact(caches=caches)
            plain.compact(1 << 30)
            check_pool(pool, plain)
        for c, was in zip(caches, before):
            now = contents(c, pool.page_table, plain.lens, ps)
            for i in range(batch):
                for x, y in zip(now[i], was[parents[i]] if kept[i] else now[i]):
                    assert torch.equal(x[:kept[i]], y[:kept[i]]), (turn, i)
            for i in range(batch):                                   # new tokens of its own for every row
                for at in range(kept[i], plain.lens[i]):
                    page = int(pool.page_table[i, at // ps])
                    fresh = torch.randn(h, d, device="cuda")
                    c.k[page, :, at % ps], c.v[page, :, at % ps] = fresh.to(dtype), (-fresh).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("layouts", [("pages", "pages"), ("tokens", "heads"), ("padded", "tokens"), ("heads", "padded")])
def test_copies_between_caches(dtype, d, layouts):
    h, ps = 3, 8
    raw = torch.int16 if dtype == BF else torch.uint8
    for n_from, n_to in ((12, 12), (5, 40)):
        frm = [S.PagedCache(page_arrays(n_from, h, ps, d, dtype, layouts[0], l), page_arrays(n_from, h, ps, d, dtype, layouts[0], 50 + l), ints([[0]])) for l in range(2)]
        to = [S.PagedCache(page_arrays(n_to, h, ps, d, dtype, layouts[1], 20 + l), page_arrays(n_to, h, ps, d, dtype, layouts[1], 70 + l), ints([[0]])) for l in range(2)]
        src, dst, rows = [3, 0, n_from, 1, 1, -1, 2, 4], [4, 1, 0, n_to, 2, 3, n_to - 1, 6], [8, 3, 8, 8, 0, 8, 99, -4]
        for use_rows in (False, True):
            want = [(c.k.clone(), c.v.clone()) for c in to]
            for c, (wk, wv) in zip(frm, want):
                for s, t, r in zip(src, dst, rows):
                    if 0 <= s < n_from and 0 <= t < n_to:
                        m = min(max(r, 0), ps) if use_rows else ps
                        wk[t, :, :m], wv[t, :, :m] = c.k[s, :, :m], c.v[s, :, :m]
            S.pages_copy(frm, ints(src), ints(dst), ints(rows) if use_rows else None, to=to)
            for c, (wk, wv) in zip(to, want):
                assert torch.equal(c.k.contiguous().view(raw), wk.contiguous().view(raw)) and torch.equal(c.v.contiguous().view(raw), wv.contiguous().view(raw))


def test_copies_of_many_layers_of_several_shapes():
    caches = []
    for l in range(75):
        h, d, n = [(2, 64, 9), (1, 128, 9), (2, 64, 7)][l // 35]
        caches.append(S.PagedCache(page_arrays(n, h, 16, d, BF, "pages", l), page_arrays(n, h, 16, d, BF, "pages", 100 + l), ints([[0]])))
    want = [(c.k.clone(), c.v.clone()) for c in caches]
    for wk, wv in want:
        for s, t in ((0, 5), (1, 6), (8, 3)):
            if s < len(wk):
                wk[t], wv[t] = wk[s], wv[s]
    S.pages_copy(caches, ints([0, 1, 8]), ints([5, 6, 3]))
    assert all(torch.equal(c.k, wk) and torch.equal(c.v, wv) for c, (wk, wv) in zip(caches, want))
    S.pages_copy(caches, ints([]), ints([]))
    S.pages_copy([], ints([0]), ints([1]))
    with pytest.raises(S.ShadowKVError):
        S.pages_copy(caches[:1], ints([0]), ints([1]), to=caches[40:41])


def test_a_page_beyond_four_gib():
    h, ps, d = 8, 1024, 128
    n = 2 ** 32 // (h * ps * d * 2) + 9
    k = torch.zeros(n, h, ps, d, dtype=BF, device="cuda")
    v = torch.zeros(n, h, ps, d, dtype=BF, device="cuda")
    k[3], v[3] = 1.5, 2.5
    cache = S.PagedCache(k, v, ints([[0]]))
    S.pages_copy(cache, ints([3]), ints([n - 1]))
    S.pages_copy(cache, ints([n - 1]), ints([5]))
    assert bool((k[n - 1] == 1.5).all()) and bool((v[5] == 2.5).all()) and float(k[n - 2].abs().sum()) == 0.0


@pytest.mark.parametrize("batch", [5, 1500])
def test_tables_with_a_stride_and_counts_at_any_address(batch):
    """The C interface's pool: rows of the table further apart than they are long, counts that are aligned to themselves only; what lies
    between the rows is left alone."""
    width, n_pages, ps = 6, 40 + 4 * batch, 4
    pool, plain = S.PagePool(batch, width, n_pages, ps), PlainPool(batch, width, n_pages, ps)
    wide = torch.full((batch, width + 3), 77, dtype=torch.int32, device="cuda")
    pool.page_table = wide[:, :width].fill_(-1)
    pool.page_refs = torch.full((n_pages + 2,), 0, dtype=torch.int32, device="cuda")[1:-1]
    c = pool._c._obj
    c.page_table, c.table_stride, c.page_refs = wide.data_ptr(), width + 3, pool.page_refs.data_ptr()
    rng = random.Random(batch)
    for turn in range(4):
        step(pool, plain, [rng.randint(-1, batch - 1) for _ in range(batch)] if turn else None, None, [rng.randint(0, 9) for _ in range(batch)])
        if turn % 2:
            pool.compact()
            plain.compact(1 << 30)
            check_pool(pool, plain)
    assert bool((wide[:, width:] == 77).all())


def test_a_large_pool():
    n_pages, ps = 300001, 4
    pool, plain = S.PagePool(8, 60000, n_pages, ps), PlainPool(8, 60000, n_pages, ps)
    gen = torch.Generator().manual_seed(5)
    busy = torch.rand(n_pages, generator=gen) < 0.6
    plain.refs = busy.int().tolist()                                 # held by others
    put_pool(pool, plain)
    step(pool, plain, n_new=[70001, 5, 100000, 0, 33333, 1, 1, 90000])
    step(pool, plain, [2, 2, 0, 1, 0, -1, 6, 4], None, 3)
    for most in (1000, None):
        used = pool.compact(max_moves=most)
        moves, end = plain.compact(1 << 30 if most is None else most)
        check_pool(pool, plain)
        assert int(used) == end and [m[:2] for m in moves_of(pool)] == moves


def test_a_captured_step():
    batch, width, n_pages, ps = 8, 20, 120, 4
    pool, plain = S.PagePool(batch, width, n_pages, ps), PlainPool(batch, width, n_pages, ps)
    k, v = (page_arrays(n_pages, 2, ps, 64, BF, "pages", i) for i in range(2))
    cache = pool.cache(k, v)
    parents, grow = ints(list(range(batch))), ints([5] * batch)
    step(pool, plain, n_new=[5] * batch, caches=cache)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.update(parents=parents, n_new=grow, caches=cache)
        used = pool.compact(max_moves=3, caches=cache)
    check_pool(pool, plain)                                          # capturing does nothing
    rng = random.Random(11)
    for _ in range(6):
        p, g = [rng.randint(-1, batch - 1) for _ in range(batch)], [rng.randint(0, 6) for _ in range(batch)]
        parents.copy_(ints(p))
        grow.copy_(ints(g))
        before = contents(cache, pool.page_table, plain.lens, ps)
        graph.replay()
        torch.cuda.synchronize()
        _, kept = plain.update(p, None, g)
        _, end = plain.compact(3)
        check_pool(pool, plain)
        assert int(used) == end
        now = contents(cache, pool.page_table, plain.lens, ps)
        assert all(torch.equal(now[i][0][:kept[i]], before[p[i]][0][:kept[i]]) for i in range(batch) if kept[i])


def test_another_stream():
    pool, plain = S.PagePool(3, 5, 20, 4), PlainPool(3, 5, 20, 4)
    cache = pool.cache(*(page_arrays(20, 1, 4, 64, BF, "pages", i) for i in range(2)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    parents = ints([0, 0, 0])
    side.wait_stream(torch.cuda.current_stream())
    pool.update(n_new=6, caches=cache, stream=side)
    pool.update(parents=parents, n_new=1, caches=cache, stream=side)
    side.synchronize()
    plain.update(None, None, 6)
    plain.update([0, 0, 0], None, 1)
    check_pool(pool, plain)
    with pytest.raises(ValueError):
        S.PagePool(3, 5, 21, 4).update(caches=cache)
