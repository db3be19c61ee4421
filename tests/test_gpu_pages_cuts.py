"""Rows that stay where they are and give up pages: a few, which one thread takes back, and many, which go with the rows that move."""
import random

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import PlainPool, check_pool, moves_of

pytestmark = pytest.mark.gpu


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("batch,width,ps", [(1, 40, 4), (5, 33, 1), (64, 64, 8), (7, 9000, 2), (1000, 30, 4), (3, 30000, 4)])
def test_cuts_of_all_lengths(batch, width, ps):
    """Rows cut by 0 to all of their pages, in one call with rows that continue what is cut, that are emptied, and that grow."""
    rng = random.Random(batch + width)
    n_pages = batch * width + 9
    pool, plain = S.PagePool(batch, width, n_pages, ps), PlainPool(batch, width, n_pages, ps)
    for turn in range(6):
        full = [width * ps - rng.randint(0, 3 * ps) if width * ps > 3 * ps else 0 for _ in range(batch)]
        grow = [max(f - n, 0) for f, n in zip(full, plain.lens)]
        keep = [rng.choice([0, 1, ps, max(n - rng.randint(0, 40 * ps), 0), rng.randint(0, max(n, 1)), n]) for n in full]
        stays = rng.choice([1.0, 0.7])
        parents = None if turn % 3 == 0 else [i if rng.random() < stays else rng.randint(-1, batch - 1) for i in range(batch)]
        for args in ((None, None, grow), (parents, keep, rng.choice([0, 1, ps + 1]))):
            pool.update(ints(args[0]), ints(args[1]), args[2] if isinstance(args[2], int) else ints(args[2]))
            moves, _ = plain.update(*args)
            check_pool(pool, plain)
            assert moves_of(pool) == moves


@pytest.mark.parametrize("batch,width", [(1, 65536), (8, 8192)])
def test_a_long_cut_takes_no_longer_than_freeing_the_row(batch, width):
    """The same pages given up through keep_lens and through a parent outside the batch.  (One after the other by a thread a row, 65536 take 600 times as long.)"""
    pool = S.PagePool(batch, width, batch * width, 16)
    ways = {"cut": dict(keep_lens=ints([0] * batch)), "freed": dict(parents=ints([-1] * batch))}
    took = {k: [] for k in ways}
    for _ in range(6):
        for name, kw in ways.items():
            pool.page_table.copy_(torch.arange(batch * width, device="cuda", dtype=torch.int32).view(batch, width))
            pool.kv_lens.fill_(width * 16)
            pool.page_refs.fill_(1)
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            torch.cuda.synchronize()
            start.record()
            pool.update(**kw)
            end.record()
            torch.cuda.synchronize()
            took[name].append(start.elapsed_time(end))
            assert int(pool.page_refs.abs().sum()) == 0 and int(pool.kv_lens.sum()) == 0 and bool((pool.page_table == -1).all())
    assert min(took["cut"]) <= 20 * min(took["freed"]), took
