"""Captured calls on the paged cache whose page table, lengths, run boundaries and inputs change between replays."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8, Cache

pytestmark = pytest.mark.gpu


def _x(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,t", [(BF, 3), (F8, 3), (BF, 90)])
def test_replays_follow_the_page_table(dtype, t):
    """Every replay finds its pages anew, entries without a page among them: as an eager call on a copy of the cache of before."""
    d, hq, hkv, page, width, n_pages = 64, 8, 2, 16, 20, 60
    pages = Cache([0] * 3, hkv, d, dtype, page, spare=n_pages, width=width)
    raw = {BF: torch.int16, F8: torch.uint8}[dtype]
    for x in (pages.k, pages.v):
        x.view(raw).zero_()
    table = torch.zeros(3, width, dtype=torch.int32, device="cuda")
    c = S.PagedCache(pages.k, pages.v, table)
    lens, starts = torch.ones(3, dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    k, v, q = _x(1, BF, t, hkv, d), _x(2, BF, t, hkv, d), _x(3, BF, t, hq, d)
    rope = S.Rope(d)
    ws = torch.empty(S.paged_attention_workspace_bytes(c, hq, t), dtype=torch.uint8, device="cuda")
    out = torch.zeros(t, hq, d, dtype=BF, device="cuda")
    rotated = torch.empty_like(q)

    def step(cache, w, o, qq):
        S.paged_append(cache, k, v, lens, seq_starts=starts, rope=rope, q=q, q_out=qq)
        return S.paged_attention(cache, qq, lens, seq_starts=starts, workspace=w, out=o)
    step(c, ws, out, rotated)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c, ws, out, rotated)
    gen = torch.Generator().manual_seed(5)
    seen = []
    for i in range(8):
        now = torch.randperm(n_pages, generator=gen).int().view(3, width)
        now[torch.rand(3, width, generator=gen) < 0.1] = -1
        table.copy_(now)
        news = [t // 3 - i % 2, t // 3, t - 2 * (t // 3) - i % 3 // 2]
        starts.copy_(torch.tensor([0, news[0], news[0] + news[1], sum(news)], dtype=torch.int32))
        lens.copy_(torch.tensor([max(news[0], 1) + 30 * i, news[1] + 7, 320 - i], dtype=torch.int32))
        for x, seed in ((k, i), (v, 50 + i), (q, 90 + i)):
            x.copy_(_x(seed, BF, *x.shape))
        before = S.PagedCache(pages.k.clone(), pages.v.clone(), table.clone())
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want, want_q = torch.full_like(out, 7.0), torch.empty_like(rotated)
        step(before, None, want, want_q)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(rotated[:sum(news)], want_q[:sum(news)])
        assert torch.equal(pages.k.view(raw), before.k.view(raw)) and torch.equal(pages.v.view(raw), before.v.view(raw))
        assert (out[sum(news):] == 7).all()
        seen.append(out.clone())
    assert not any(torch.equal(a, b) for a, b in zip(seen, seen[1:]))
