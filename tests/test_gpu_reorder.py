"""Rows of dense state arrays that follow their parents, in place: what comes out is what went in, element by element."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S

pytestmark = pytest.mark.gpu


def want_of(x, parents):
    n = x.shape[0]
    p = parents.reshape(-1).long().cpu()
    return x[torch.where((p >= 0) & (p < n), p, torch.arange(n)).to(x.device)].clone()


def raw(t):
    return t.contiguous().view(torch.uint8) if t.dim() and t.numel() else t


def check(arrays, parents, **kw):
    want = [want_of(x, parents) for x in arrays]
    S.reorder_rows(arrays, parents, **kw)
    torch.cuda.synchronize()
    for x, w in zip(arrays, want):
        assert torch.equal(raw(x), raw(w)), (tuple(x.shape), x.dtype)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rand(shape, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = torch.empty(shape, dtype=dtype, device="meta").numel() * torch.empty((), dtype=dtype).element_size()
    return torch.randint(0, 256, (n,), generator=gen, device="cuda", dtype=torch.uint8).view(dtype).view(shape)


@pytest.mark.parametrize("parents", [[0], [0, 0, 0, 0], [1, 0, 3, 2], [1, 2, 3, 0], [3, 3, 1, 1], [0, 1, 2, 3], [-1, 0, 7, 1], [2, 2, 2, 2],
                                     [1, 2, 3, 4, 5, 6, 0, 0], [6, 5, 4, 3, 2, 1, 0, -5, 2 ** 31 - 1]])
@pytest.mark.parametrize("shape,dtype", [((8, 32, 128), torch.bfloat16), ((515,), torch.int32), ((), torch.float32), ((3, 7), torch.uint8),
                                         ((13,), torch.int16), ((2, 9, 16), torch.float8_e5m2), ((5000,), torch.int64)])
def test_parents_and_types(parents, shape, dtype):
    check([rand((len(parents), *shape), dtype)], ints(parents))


@pytest.mark.parametrize("n,moved", [(2, 1), (64, 5), (255, 255), (256, 200), (257, 3), (1000, 1000), (2048, 2048), (2048, 17)])
def test_rows(n, moved):
    gen = torch.Generator().manual_seed(n + moved)
    parents = torch.arange(n, dtype=torch.int32)
    which = torch.randperm(n, generator=gen)[:moved]
    parents[which] = torch.randint(-1, n + 1, (moved,), generator=gen, dtype=torch.int32)
    check([rand((n, 1003), torch.int16, 1), rand((n, 64), torch.bfloat16, 2), rand((n,), torch.int32, 3)], parents.cuda())


def test_views():
    x = rand((6, 4, 100, 32), torch.bfloat16)
    before = x.clone()
    p = ints([[1, 0, 2], [5, 5, 3]])
    views = (lambda t: t[:, :, 60:], lambda t: t[:, 1:3, :10], lambda t: t[:, 3, 20:30], lambda t: t[:, 0, :, 16:], lambda t: t[:, 2, ::2, 1:3])
    for view in views:
        w = want_of(view(before), p)
        S.reorder_rows(view(x), p)
        want = before.clone()
        view(want).copy_(w)
        assert torch.equal(raw(x), raw(want))                        # and nothing else has changed
        before = x.clone()
    kv = rand((6, 2, 50, 8), torch.bfloat16)
    w = want_of(kv, p)
    S.reorder_rows([kv[:, 0], kv[:, 1]], p)                          # arrays that interleave
    assert torch.equal(raw(kv), raw(w))
    t = rand((50, 6, 8), torch.int32)
    w = want_of(t.transpose(0, 1), p)
    S.reorder_rows(t.transpose(0, 1), p)                             # rows inside
    assert torch.equal(t.transpose(0, 1), w)
    with pytest.raises(ValueError):
        S.reorder_rows(x[:, ::2, ::2], p)
    with pytest.raises(ValueError):
        S.reorder_rows(x[:5], p)
    with pytest.raises(S.ShadowKVError):
        S.reorder_rows([x, x], p)
    with pytest.raises(S.ShadowKVError):
        S.reorder_rows(x[:1].expand(6, 4, 100, 32), p)


def test_many_arrays_of_all_kinds():
    gen = torch.Generator().manual_seed(4)
    parents = torch.randint(0, 12, (12,), generator=gen, dtype=torch.int32).cuda()
    arrays = []
    for i in range(150):
        dtype = [torch.bfloat16, torch.int32, torch.uint8, torch.float32][i % 4]
        arrays.append(rand((12, *[(3,), (0,), (16, 8), (1 + 37 * i,)][i // 4 % 4]), dtype, i))
    check(arrays, parents)
    S.reorder_rows([], parents)
    S.reorder_rows([torch.empty(0, 5, device="cuda")], ints([]))


def test_a_row_beyond_four_gib():
    x = torch.zeros(3, 2 ** 32 + 48, dtype=torch.uint8, device="cuda")
    x[:, -48:] = rand((3, 48), torch.uint8)
    x[:, :48] = rand((3, 48), torch.uint8, 1)
    head, tail = x[:, :48].clone(), x[:, -48:].clone()
    S.reorder_rows(x, ints([2, 0, 0]))
    for part, was in ((x[:, :48], head), (x[:, -48:], tail)):
        assert torch.equal(part, was[[2, 0, 0]])


def test_another_stream_and_captured_calls():
    x, p = rand((16, 1000), torch.int32), ints([0] * 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = want_of(x, p)
    S.reorder_rows(x, p, stream=side)
    side.synchronize()
    assert torch.equal(x, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.reorder_rows(x, p)
    gen = torch.Generator().manual_seed(7)
    for seed in range(4):
        x.copy_(rand((16, 1000), torch.int32, seed))
        p.copy_(torch.randint(-1, 16, (16,), generator=gen, dtype=torch.int32))
        want = want_of(x, p)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want)
