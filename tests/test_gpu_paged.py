"""shadowkv_paged_append and shadowkv_paged_attention against their plain forms in 64 bits.  Whatever a call must not look at
is NaN: rows behind a sequence's end, unused pages."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, F8, Cache, attention, check_attention, check_turned

pytestmark = pytest.mark.gpu


def _q(n, hq, d, seed=1):
    return torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


def _attend(cache, q, news, causal=True, **kw):
    lse = torch.full(q.shape[:2], 123.0, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts(news), causal=causal, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


# sequences as (new tokens, length with them)
ONE = [[(1, 1)], [(1, 31), (1, 32), (1, 33)], [(1, 1000)], [(1, 5003), (0, 40), (1, 2), (1, 129)], [(1, 20000)]]
FEW = [[(3, 3), (5, 700)], [(0, 0), (2, 128), (4, 4097), (1, 65), (0, 9), (3, 64)]]
MANY = [[(64, 64)], [(65, 65), (1, 300)], [(200, 200)], [(130, 1003), (0, 77), (1, 64), (257, 300)], [(700, 2900)], [(17, 17), (511, 4096)]]


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (96, 3, 3), (64, 14, 2), (128, 32, 2), (64, 32, 1), (96, 64, 1), (128, 33, 1)])
@pytest.mark.parametrize("runs", range(len(ONE) + len(FEW) + len(MANY)))
def test_attention_matches_64_bits(runs, d, hq, hkv, dtype):
    seqs = (ONE + FEW + MANY)[runs]
    news, lens = [n for n, _ in seqs], [m for _, m in seqs]
    page = [16, 64, 1, 128][(runs + hq) % 4]
    print(f"[attend] {seqs} d {d} heads {hq}/{hkv} {dtype} page {page}", flush=True)
    cache = Cache(lens, hkv, d, dtype, page, seed=runs)
    q = _q(sum(news), hq, d, seed=runs + 50)
    out, lse = _attend(cache, q, news)
    check_attention(cache, q, out, lse, news)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F8, 96)])
@pytest.mark.parametrize("seqs", [[(1, 700), (1, 3)], [(40, 700), (3, 65), (1, 0), (2, 1)], [(300, 40)]])
def test_attention_without_a_causal_mask(seqs, dtype, d):
    news, lens = [n for n, _ in seqs], [m for _, m in seqs]
    cache = Cache(lens, 2, d, dtype, 32, seed=4)
    q = _q(sum(news), 8, d)
    out, lse = _attend(cache, q, news, causal=False)
    check_attention(cache, q, out, lse, news, causal=False)


@pytest.mark.parametrize("n", [1, 5, 90])
def test_rows_that_see_nothing_are_zero(n):
    """More new tokens than the cache holds: the first ones see no key.  And no keys at all."""
    news, lens = [n, n, n], [n // 2, 0, 200 + n]
    cache = Cache(lens, 2, 128, BF, 16, seed=2)
    q = _q(sum(news), 8, 128)
    out, lse = _attend(cache, q, news)
    check_attention(cache, q, out, lse, news)
    gone = n - n // 2
    assert (out[:gone] == 0).all() and torch.isinf(lse[:gone]).all() and (out[n:2 * n] == 0).all()


@pytest.mark.parametrize("dtype,news", [(BF, [1, 1]), (F8, [3, 1]), (BF, [100, 70])])
def test_entries_without_a_page_hold_no_tokens(dtype, news):
    lens, page = [400, 300], 32
    cache = Cache(lens, 2, 128, dtype, page, seed=8)
    table = cache.table_cpu.clone()
    table[0, 0], table[0, 5], table[1, 9], table[1, 3] = -1, cache.k.shape[0], -(1 << 31), (1 << 31) - 1
    hidden = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in lens]
    for i, j in ((0, 0), (0, 5), (1, 9), (1, 3)):
        hidden[i][j * page:(j + 1) * page] = True
    cache.c = S.PagedCache(cache.k, cache.v, table.cuda())
    q = _q(sum(news), 8, 128)
    out, lse = _attend(cache, q, news)
    check_attention(cache, q, out, lse, news, hidden=hidden)
    cache.c = S.PagedCache(cache.k, cache.v, torch.full_like(table, -1).cuda())
    out, lse = _attend(cache, q, news)
    assert (out == 0).all() and torch.isinf(lse).all()


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n,hq", [(4, 8), (100, 8)])
def test_a_later_token_has_no_influence(n, hq, bad, dtype):
    """A value (and a key) that is infinite or NaN reaches the tokens that see it, and no other."""
    d, hkv, L, at = 128, 2, 300, 300 - n // 2
    cache = Cache([L], hkv, d, dtype, 16, seed=5)
    q = _q(n, hq, d)
    clean, clean_lse = _attend(cache, q, [n])
    page, row = int(cache.table_cpu[0, at // 16]), at % 16
    cache.v[page, 1, row, 5] = bad
    out, lse = _attend(cache, q, [n])
    first = at - (L - n)                     # the first token that sees it
    assert torch.equal(out[:first], clean[:first]) and torch.equal(out[:, :hq // 2], clean[:, :hq // 2])
    hit = out[first:, hq // 2:, 5].float()
    assert (torch.isnan(hit) if bad != bad else hit == bad).all()
    rest = torch.cat([out[first:, hq // 2:, :5], out[first:, hq // 2:, 6:]], -1)
    assert torch.isfinite(rest.float()).all() and torch.equal(lse, clean_lse)
    if bad != bad:
        cache.k[page, 0, row, 9] = bad
        out, lse = _attend(cache, q, [n])
        assert torch.equal(out[:first], clean[:first])
        assert torch.isnan(out[first:, :hq // 2].float()).all() and torch.isnan(lse[first:, :hq // 2]).all()


@pytest.mark.parametrize("dtype", [BF, F8])
@pytest.mark.parametrize("layout", ["tokens", "heads"])
@pytest.mark.parametrize("news", [[1, 1, 1], [70, 3, 1]])
def test_other_strides_and_padded_batches(news, layout, dtype):
    """Pages token by token or head by head; q and out in wider arrays; rows before, between and behind the runs stay."""
    lens = [200, 90, 1500]
    cache = Cache(lens, 4, 96, dtype, 64, seed=11, layout=layout, width=40)
    t = sum(news)
    wide = torch.randn(t + 9, 20, 128, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
    q = wide[:, 2:18, 16:112]
    res = torch.full((16, t + 9, 104), 7.0, dtype=BF, device="cuda")
    out = res.transpose(0, 1)[:, :, :96]
    starts = cache.starts(news) + 4
    S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=starts, out=out)
    check_attention(cache, q[4:4 + t], out[4:4 + t], None, news, rows_per_seq=(t + 9) / 3)
    assert (out[:4] == 7).all() and (out[4 + t:] == 7).all() and (res[..., 96:] == 7).all()


@pytest.mark.parametrize("seqs,hq,hkv,d,dtype", [([(32, 16738)], 14, 2, 64, F8), ([(56, 2527)], 16, 8, 64, BF), ([(1, 60000)], 16, 1, 64, BF),
                                                  ([(4, 3001), (2, 1200), (5, 4100)], 8, 2, 128, BF), ([(30, 900), (0, 9), (31, 700)], 32, 8, 96, F8),
                                                  ([(1, 1500 + i) for i in range(40)], 32, 8, 128, BF), ([(8, 33000)], 32, 8, 128, F8)])
def test_items_shared_by_a_few_or_hundreds_of_workgroups(seqs, hq, hkv, d, dtype):
    news, lens = [n for n, _ in seqs], [m for _, m in seqs]
    cache = Cache(lens, hkv, d, dtype, 64, seed=12)
    q = _q(sum(news), hq, d)
    out, lse = _attend(cache, q, news)
    check_attention(cache, q, out, lse, news)
    for fill in (0, 255):
        ws = torch.full((S.paged_attention_workspace_bytes(cache.c, hq, sum(news)),), fill, dtype=torch.uint8, device="cuda")
        again, lse2 = _attend(cache, q, news, workspace=ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_equal_runs_need_no_starts_and_results_repeat():
    cache = Cache([300, 17, 2000], 2, 64, BF, 16, seed=3)
    q = _q(12, 8, 64)
    a = S.paged_attention(cache.c, q, cache.kv_lens())
    b = S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts([4, 4, 4]))
    assert torch.equal(a, b)
    check_attention(cache, q, a, None, [4, 4, 4])
    ws = torch.full((S.paged_attention_workspace_bytes(cache.c, 8, 12),), 255, dtype=torch.uint8, device="cuda")   # NaN throughout
    for _ in range(5):
        assert torch.equal(S.paged_attention(cache.c, q, cache.kv_lens(), workspace=ws), a)


@pytest.mark.parametrize("hq,hkv,n", [(8, 2, 1), (16, 1, 2), (8, 2, 700)])
def test_many_sequences(hq, hkv, n):
    """More sequences than a workgroup has threads, most of them with nothing to do."""
    b = 600
    news = [0] * b
    for i in (0, 3, 255, 256, 257, 511, 512, 599):
        news[i] = n if i == 512 else 1
    lens = [(i * 37) % 90 + max(1, m) for i, m in enumerate(news)]
    cache = Cache(lens, hkv, 64, BF, 16, seed=9)
    q = _q(sum(news), hq, 64)
    out, lse = _attend(cache, q, news)
    check_attention(cache, q, out, lse, news)


def test_logits_far_apart_and_extreme_scales():
    """Logits up to thousands: weights underflow, the maximum moves by more than fp32's exponents hold at once."""
    cache = Cache([2000, 64], 2, 128, BF, 64, seed=6, k_gain=60.0)
    for news in ([1, 1], [64, 64]):
        q = _q(sum(news), 8, 128) * 4
        out, lse = _attend(cache, q, news)
        check_attention(cache, q, out, lse, news)
        out, lse = _attend(cache, q, news, softmax_scale=1e-4)
        check_attention(cache, q, out, lse, news, scale=1e-4)


# ---- append ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kt,ct", [(BF, BF), (BF, F8), (F8, F8)])
@pytest.mark.parametrize("d,rot,layout", [(128, 0, 0), (96, 24, 1), (64, 32, 0), (96, 0, 1)])
@pytest.mark.parametrize("seqs", [[(1, 1)], [(1, 500), (1, 1), (0, 20), (1, 65)], [(130, 130), (0, 0), (45, 300), (1, 64)]])
def test_append_matches_64_bits(seqs, d, rot, layout, kt, ct):
    news, lens = [n for n, _ in seqs], [m for _, m in seqs]
    print(f"[append] {seqs} d {d} rot {rot} {layout} {kt} {ct}", flush=True)
    hkv, hq, page, t = 3, 6, 32, sum(news)
    cache = Cache(lens, hkv, d, ct, page, seed=1)
    r = S.Rope(d, rot_dim=rot, layout=layout, theta=1e4)
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = ((torch.randn(t, hkv, d, generator=gen, device="cuda") * 2).to(kt) for _ in range(2))
    q = _q(t, hq, d)
    off = torch.tensor([7 * i for i in range(len(seqs))], dtype=torch.int32, device="cuda")
    before_k, before_v = cache.k.clone(), cache.v.clone()
    q_out = S.paged_append(cache.c, k, v, cache.kv_lens(), seq_starts=cache.starts(news), rope=r, q=q, pos_offset=off)
    torch.cuda.synchronize()
    place = torch.cat([torch.arange(m - n, m) for n, m in seqs]).cuda()
    seq = torch.cat([torch.full((n,), i) for i, (n, _) in enumerate(seqs)]).long().cuda()
    pos = place + off[seq]
    check_turned(r, q_out, q, pos)
    pg = cache.table[seq, place // page].long()
    raw = {BF: torch.int16, F8: torch.uint8}[ct]
    kr, vr = cache.k.view(raw)[pg, :, place % page].view(ct), cache.v.view(raw)[pg, :, place % page].view(ct)
    check_turned(r, kr, k, pos)
    assert torch.equal(vr.view(raw), v.to(ct).view(raw))
    for now, was in ((cache.k, before_k), (cache.v, before_v)):      # nothing else is touched
        now, was = now.view(raw).clone(), was.view(raw)
        now[pg, :, place % page] = was[pg, :, place % page]
        assert torch.equal(now, was)


def test_append_without_rotation_in_place_queries_and_dropped_places():
    d, hkv, page = 128, 2, 16
    cache = Cache([40, 3, 64], hkv, d, BF, page, seed=3)
    raw_k = cache.k.clone()
    t = 30
    k, v, q = _q(t, hkv, d, 1), _q(t, hkv, d, 2), _q(t, 4, d, 3)
    # sequence 0: places 30..39; 1: three of its ten places are below zero... 7 of 10; 2: the last six lie beyond its pages
    lens = torch.tensor([40, 3, 70], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 10, 20, 30], dtype=torch.int32, device="cuda")
    S.paged_append(cache.c, k, v, lens, seq_starts=starts)
    got = cache.k.clone()
    for i, (first, n) in enumerate(((30, 10), (-7, 10), (60, 10))):
        for j in range(n):
            p = first + j
            if 0 <= p < 64 and p // page < cache.table.shape[1] and int(cache.table_cpu[i, p // page]) >= 0:
                raw_k[int(cache.table_cpu[i, p // page]), :, p % page] = k[10 * i + j]
    assert torch.equal(got.view(torch.int16), raw_k.view(torch.int16))
    r = S.Rope(d)
    want = S.paged_append(cache.c, k, v, lens, seq_starts=starts, rope=r, q=q)
    mine = q.clone()
    assert S.paged_append(cache.c, k, v, lens, seq_starts=starts, rope=r, q=mine, q_out=mine) is mine
    assert torch.equal(mine, want)
    check_turned(r, want, q, torch.cat([torch.arange(30, 40), torch.arange(-7, 3), torch.arange(60, 70)]).cuda())


def test_append_leaves_rows_outside_the_runs():
    d, hkv = 64, 2
    cache = Cache([20] * 3, hkv, d, BF, 16, seed=3)
    k, v, q = _q(12, hkv, d, 1), _q(12, hkv, d, 2), _q(12, 4, d, 3)
    q_out = torch.full_like(q, 9.0)
    starts = torch.tensor([2, 5, 5, 9], dtype=torch.int32, device="cuda")
    S.paged_append(cache.c, k, v, cache.kv_lens(), seq_starts=starts, rope=S.Rope(d), q=q, q_out=q_out)
    assert (q_out[:2] == 9).all() and (q_out[9:] == 9).all() and not (q_out[2:9] == 9).all()
    check_turned(S.Rope(d), q_out[2:9], q[2:9], torch.tensor([17, 18, 19, 16, 17, 18, 19]).cuda())


def test_append_values_round_as_the_storage_type_does():
    """Every bf16 number, as value and as key without rotation, against torch's cast."""
    d, page = 128, 256
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF).view(512, 1, d).cuda()
    cache = Cache([512], 1, d, F8, page, seed=1)
    S.paged_append(cache.c, bits, bits, cache.kv_lens())
    want = bits.to(F8)
    for store in (cache.k, cache.v):
        got = store.view(torch.uint8)[cache.table[0].long()].view(F8).reshape(512, 1, d)
        nan = torch.isnan(bits.float())
        assert torch.equal(torch.isnan(got.float()), nan)
        assert torch.equal(got.view(torch.uint8)[~nan], want.view(torch.uint8)[~nan])


# ---- together -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F8])
def test_prompt_in_chunks_then_tokens(dtype):
    """Prompts join in chunks, then single tokens: every step's attention against the plain form over what was appended."""
    d, hq, hkv, page = 128, 8, 2, 16
    cache = Cache([0, 0], hkv, d, dtype, page, spare=30, width=14)
    order = torch.randperm(28, generator=torch.Generator().manual_seed(1)).int().view(2, 14)
    cache.table_cpu, cache.table = order, order.cuda()
    cache.c = S.PagedCache(cache.k, cache.v, cache.table)
    r = S.Rope(d, scaling=S.ROPE_BANDS, factor=8.0, low=1.0, high=4.0, original_len=64)
    lens = [0, 0]
    for step, news in enumerate(([90, 7], [60, 0], [33, 120], [1, 1], [1, 1], [0, 1], [2, 3])):
        lens = [a + b for a, b in zip(lens, news)]
        cache.lens, t = lens, sum(news)
        k, v, q = _q(t, hkv, d, 10 + step), _q(t, hkv, d, 20 + step), _q(t, hq, d, 30 + step)
        q = S.paged_append(cache.c, k, v, cache.kv_lens(), seq_starts=cache.starts(news), rope=r, q=q)
        out = S.paged_attention(cache.c, q, cache.kv_lens(), seq_starts=cache.starts(news))
        cache.kd, cache.vd = [], []
        raw = {BF: torch.int16, F8: torch.uint8}[dtype]
        for i, n in enumerate(lens):
            pl = torch.arange(n, device="cuda")
            pg = cache.table[i, pl // page].long()
            cache.kd.append(cache.k.view(raw)[pg, :, pl % page].view(dtype).double())
            cache.vd.append(cache.v.view(raw)[pg, :, pl % page].view(dtype).double())
            assert torch.isfinite(cache.kd[-1]).all()
        check_attention(cache, q, out, None, news)


def test_dense_arrays_as_pages_feed_the_sparse_path():
    """A prompt appended to dense arrays through their pages: build_landmarks finds its keys and values there, factorize_keys takes
    the keys before the rotation, and a decode step whose budget covers everything gives what attention over the pages gives."""
    b, hq, hkv, d, s = 2, 8, 2, 64, 512
    gen = torch.Generator(device="cuda").manual_seed(4)
    low = torch.randn(b, s, 32, generator=gen, device="cuda") @ torch.randn(32, hkv * d, generator=gen, device="cuda") / 6
    k_pre, v = low.to(BF), torch.randn(b, s, hkv * d, generator=gen, device="cuda").to(BF)
    k_rope, store = (torch.empty(b, hkv, s, d, dtype=BF, device="cuda") for _ in range(2))
    cache = S.dense_pages(k_rope, store, 64)
    r = S.Rope(d, theta=5e5)
    lens = torch.full((b,), s, dtype=torch.int32, device="cuda")
    S.paged_append(cache, k_pre.view(b * s, hkv, d), v.view(b * s, hkv, d), lens, rope=r)
    want = S.rotate(r, k_pre.view(b, s, hkv, d))
    assert torch.equal(k_rope, want.transpose(1, 2)) and torch.equal(store, v.view(b, s, hkv, d).transpose(1, 2))
    p = S.Params(b, hq, hkv, d, s, chunk_size=8, rank=40, n_outlier_chunks=4, topk_chunks=s // 8 - 4, local_len=0)
    pre, fac = S.build_landmarks(p, k_rope, store), S.factorize_keys(p, k_pre)
    q = _q(b, hq, d, 5)
    sparse, _, _ = S.decode_step(p, q, fac["A"], fac["B"], pre["landmarks"], pre["landmark_chunk_ids"], pre["k_outlier"],
                                 pre["v_outlier"], None, None, store)
    full = S.paged_attention(cache, q, lens, causal=False)
    # the keys have rank 32 before their rounding; A and B hold them to bf16: logits (|q||k| / 8 of about 8) off by some 2^-8 of that
    kd, vd = k_rope.double(), store.double()
    for i in range(b):
        o, _, av, size = attention(q[i:i + 1].double(), kd[i].transpose(0, 1), vd[i].transpose(0, 1), torch.tensor([s - 1]).cuda(), d ** -0.5)
        assert ((full[i:i + 1].double() - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -16 + 2.0 ** -17 * size[..., None] + 2.0 ** -20) * 1.01 * av).all()
        assert ((sparse[i:i + 1].double() - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -6 * size[..., None] * av).all()


def test_captured_and_replayed_with_changing_lengths():
    """Append and attention in a graph; the lengths, the table and the inputs change between replays, eager calls in between; two
    graphs with a workspace each."""
    d, hq, hkv, page = 128, 8, 2, 16
    cache = Cache([50, 200, 31], hkv, d, BF, page, seed=2, width=20, spare=40)
    table = torch.arange(60, dtype=torch.int32).view(3, 20)[:, torch.randperm(20, generator=torch.Generator().manual_seed(2))].contiguous()
    pages = Cache([0] * 3, hkv, d, BF, page, spare=60, width=20)
    pages.k.zero_()
    pages.v.zero_()
    c = S.PagedCache(pages.k, pages.v, table.cuda())
    lens = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")
    k, v, q = _q(3, hkv, d, 1), _q(3, hkv, d, 2), _q(3, hq, d, 3)
    r = S.Rope(d)
    ws = [torch.empty(S.paged_attention_workspace_bytes(c, hq, 3), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(w):
        qq = S.paged_append(c, k, v, lens, rope=r, q=q)
        return S.paged_attention(c, qq, lens, workspace=w)
    step(ws[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for w in ws:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(w))
        graphs.append(g)
    for i in range(12):
        lens.copy_(torch.tensor([1 + 7 * i, 1 + 20 * i, 320 - i], dtype=torch.int32))
        for x, seed in ((k, i), (v, 50 + i), (q, 90 + i)):
            x.copy_(_q(*x.shape, seed=seed))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = outs[i % 2].clone()
        assert torch.equal(got, step(None))
        torch.cuda.synchronize()
