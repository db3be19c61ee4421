"""The choice over beams and vocabulary against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from search_util import LOGIT_TYPES, check_choice, choose

pytestmark = pytest.mark.gpu


def draw(groups, beams, vocab, dtype, seed, std=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(groups, beams, vocab, generator=gen, device="cuda") * std).to(LOGIT_TYPES[dtype])
    s = -10.0 * torch.rand(groups, beams, generator=gen, device="cuda")
    return x, s, gen


def both(x, s, n=0, slack=0.0, **kw):
    got = S.beam_select(x, s, n_out=n, **kw)
    want = choose(x, s.cpu(), n or x.shape[1], kw.get("finished"), kw.get("lengths"), kw.get("length_penalty", 0.0), kw.get("logit_scale", 0.0) or 1.0,
                  kw.get("end_token", -1))
    check_choice(got, want, slack)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("groups,beams,vocab,n", [(1, 1, 1, 1), (2, 3, 1, 4), (3, 2, 7, 5), (1, 4, 511, 4), (2, 4, 512, 8), (2, 5, 513, 5), (1, 3, 2047, 6),
                                                  (1, 3, 2048, 64), (2, 2, 2049, 64), (3, 64, 1000, 64), (1, 33, 4101, 33), (5, 4, 50257, 8), (1, 2, 300001, 2)])
def test_sizes(dtype, groups, beams, vocab, n):
    x, s, _ = draw(groups, beams, vocab, dtype, groups * 1000 + vocab)
    both(x, s, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_strides_and_addresses(dtype):
    x, s, _ = draw(4, 6, 1003, dtype, 5)
    both(x[:, 1:5, :997], s[:, 1:5].contiguous())                    # a padded vocabulary, some of the beams
    both(x.transpose(0, 1), s.t().contiguous())                      # beams outside
    both(x[..., 1:], s, 7)                                           # rows that begin at any element
    both(x[:1].expand(3, 6, 1003), s[:3].contiguous())               # groups that share their logits
    flat = torch.randn(20000, device="cuda").to(LOGIT_TYPES[dtype])
    both(flat.as_strided((2, 3, 600), (5, 301, 1), 3), torch.zeros(2, 3, device="cuda"))   # rows inside each other


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_ties_go_to_the_lower_row_and_token(dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    row = torch.randint(-2, 3, (1, 1, 3001), generator=gen, device="cuda").to(LOGIT_TYPES[dtype])
    x, s = row.expand(2, 8, 3001).contiguous(), torch.zeros(2, 8, device="cuda")
    both(x, s, 64)
    both(torch.zeros_like(x), s, 64)
    both(x[:, :4], s[:, :4].contiguous(), 4)
    both(torch.zeros_like(x)[:, :4], s[:, :4].contiguous(), 4)
    s[:, 3] = 1.0
    both(x, s, 13)
    assert both(torch.full_like(x, -0.0), s, 5)["tokens"][0].tolist() == [0, 1, 2, 3, 4]
    mixed = torch.zeros_like(x)
    mixed[..., ::2] = -0.0                                           # both zeros are one logit
    assert both(mixed, s, 5)["tokens"][0].tolist() == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("n", [1, 4, 8, 64])
def test_sorted_rows(n):
    up = torch.arange(20000, device="cuda", dtype=torch.float32) * 1e-3
    x = torch.stack([up, up.flip(0), up.roll(9999)])[None]
    both(x, torch.zeros(1, 3, device="cuda"), n)


def test_rows_that_offer_nothing():
    x, s, _ = draw(5, 6, 2500, "fp32", 9)
    s[0, 1], s[0, 2], s[0, 3], s[1] = -math.inf, math.nan, math.inf, -math.inf
    x[2, 0, 77], x[2, 1, 2499], x[2, 2, 0], x[2, 3] = math.nan, math.inf, -math.nan, -math.inf
    x[3], x[3, 2, 1999], x[3, 4, 5:8] = -math.inf, 1.0, torch.tensor([3.0, -9.0, 2.0], device="cuda")
    x[4, :, 100:] = -math.inf
    got = both(x, s, 8)
    assert got["parents"][1].tolist() == [-1] * 8 and got["parents"][3].tolist()[4:] == [-1] * 4
    for dtype in ("bf16", "fp16"):
        both(x.to(LOGIT_TYPES[dtype]), s, 8)
    first = torch.full((5, 6), -math.inf, device="cuda")
    first[:, 0] = 0.0
    assert (both(x[4:].expand(5, 6, 2500).contiguous(), first)["parents"] == 6 * torch.arange(5, device="cuda")[:, None]).all()


def test_infinite_parts_beside_finite_ones():
    x, s, _ = draw(1, 4, 9000, "fp32", 11)
    x[0, 0, :8000], x[0, 1, 600:], x[0, 2, 10:8999], x[0, 3, 1:] = -math.inf, -math.inf, -math.inf, -math.inf
    both(x, s, 16)


@pytest.mark.parametrize("groups,beams,n", [(2, 3, 4), (2, 3, 6), (1, 6, 20)])
def test_masks_that_leave_few_blocks(groups, beams, n):
    """All that is left of a row lies side by side: fewer stretches of it than places, each of them full."""
    x, s, _ = draw(groups, beams, 30000, "bf16", 21)
    x[..., :7000], x[..., 7900:] = -math.inf, -math.inf
    both(x, s, n)
    x[0, 0, 7001:], x[0, 1, :7899] = -math.inf, -math.inf
    both(x, s, n)
    x[0, 2, 7000:7900] = 1.0
    both(x, s, n)


@pytest.mark.parametrize("n", [4, 6])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_very_low_logits(dtype, n):
    """Nothing but logits far below zero: the row's sum is of what they are relative to the largest, whatever that is.  Thousands of rows, for
    what depends on the lowest bits of a product."""
    for seed, scale in enumerate((1.0, 0.7, 1.9)):
        gen = torch.Generator(device="cuda").manual_seed(40 + seed)
        x = (-10.0 ** (3.0 + 35.0 * torch.rand(3000, 4, 1, generator=gen, device="cuda"))).to(LOGIT_TYPES[dtype]).repeat(1, 1, 33)
        x[1000:1500, :, 20:], x[1500:2000, :, 5:9] = -math.inf, torch.finfo(x.dtype).min
        both(x, torch.zeros(3000, 4, device="cuda"), n, logit_scale=scale)


@pytest.mark.parametrize("n", [4, 6])
@pytest.mark.parametrize("scale", [1.0, 1.29, 1.31, 2.7])
def test_large_logits_a_step_apart(n, scale):
    """Around 2^32 fp32 has steps of 512: the next larger logit weighs up to 2^960 times as much, more than that moves the reference."""
    x = torch.full((3, 4, 6000), 2.0 ** 32, device="cuda")
    x[0, :, 1000:] += 512.0
    x[1, 1:, ::7] += 512.0
    x[1, 2:, 5000:5100] += 1024.0
    x[2, :, 3000:] = -(2.0 ** 32)
    x[2, 1:, 100:4000:3] = -math.inf
    both(x, -torch.arange(12, device="cuda", dtype=torch.float32).view(3, 4), n, slack=2.0 ** -50 * 2.0 ** 33, logit_scale=scale)


def test_masks_of_the_lowest_value():
    for dtype in ("bf16", "fp16", "fp32"):
        x, s, _ = draw(2, 4, 5000, dtype, 12)
        low = torch.finfo(x.dtype).min
        x[0, :, 3:] = low                                            # fewer left than are asked for
        x[1, 0], x[1, 1, 0:4999], x[1, 2, 1:] = low, low, low        # every token of a row: all alike
        both(x, s, 6)
        both(x, s, 4)
        both(x, s, 6, logit_scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_logits_too_small_to_be_normal(dtype):
    x = torch.zeros(1, 3, 4000, device="cuda").to(LOGIT_TYPES[dtype])
    bits = x.view(torch.int32 if dtype == "fp32" else torch.int16)
    bits[0, 0, 100:105] = torch.tensor([1, 3, 2, 3, 5], device="cuda").to(bits.dtype)
    bits[0, 1, 7] = 4
    x[0, 2] = -1.0
    got = both(x, torch.tensor([[0.0, -1.0, -2.0]], device="cuda"), 7)
    assert got["tokens"][0].tolist() == [104, 101, 103, 102, 100, 0, 1]


def test_a_temperature_that_leaves_nothing_but_ties():
    x, _, _ = draw(2, 3, 999, "fp32", 19)
    both(x, torch.zeros(2, 3, device="cuda"), 6, logit_scale=1e-30)


def test_how_many_rows_a_call_has_changes_its_sums_in_their_last_bits_only():
    x, s, _ = draw(40, 4, 70000, "bf16", 20)
    all_of_them = S.beam_select(x, s, n_out=4)
    for g in (0, 39):
        one = S.beam_select(x[g:g + 1], s[g:g + 1], n_out=4)
        assert torch.equal(one["tokens"][0], all_of_them["tokens"][g]) and torch.equal(one["parents"][0] + 4 * g, all_of_them["parents"][g])
        assert ((one["scores"][0] - all_of_them["scores"][g]).abs() <= 2.0 ** -23 * one["scores"][0].abs()).all()


def test_logits_far_apart():
    x, s, _ = draw(1, 5, 7000, "fp32", 13)
    x[0, 0, 3000:] += 2e4                                            # a part far above those before it
    x[0, 1, :3000] += 2e4
    x[0, 2] *= 1e3
    x[0, 3], x[0, 3, 6000] = -1e30, 0.0
    x[0, 4] = torch.linspace(-600, 600, 7000, device="cuda")
    both(x, s, 40, slack=2.0 ** -50 * 5e4)


@pytest.mark.parametrize("scale", [1e-3, 0.7, 1.0, 11.0])
def test_temperature(scale):
    x, s, _ = draw(3, 4, 3333, "bf16", 14)
    both(x, s, 9, logit_scale=scale, slack=2.0 ** -50 * 400)


@pytest.mark.parametrize("penalty", [0.0, 0.6, 1.0, -0.5, 16.0])
def test_ended_rows_and_lengths(penalty):
    x, s, gen = draw(6, 5, 1234, "fp16", 15)
    done = torch.rand(6, 5, generator=gen, device="cuda") < 0.4
    done[0], done[1] = True, False
    x[:, :, 700] += 25.0                                             # the end is likely
    x[0, 2] = math.nan                                               # what ended rows hold is not looked at
    s[2, :3] = -math.inf
    lens = torch.randint(0, 30, (6, 5), generator=gen, device="cuda", dtype=torch.int32)
    lens[3] = torch.tensor([0, -4, 1, 2 ** 31 - 2, 5], device="cuda", dtype=torch.int32)
    got = both(x, s, 7, finished=done, lengths=lens, length_penalty=penalty, end_token=700)
    assert got["finished"].dtype == torch.bool and bool(got["finished"][0, :5].all())
    both(x[:, 1:], s[:, 1:].contiguous(), 4, finished=done[:, 1:].contiguous(), lengths=lens[:, 1:].contiguous(), length_penalty=penalty, end_token=700)
    both(x, s, 5, finished=done)                                     # no token of its own: -1 is reported
    both(x, s, 5, end_token=1233)
    both(x, s, 5, lengths=lens)


def test_outputs_in_place_of_inputs():
    x, s, gen = draw(7, 6, 900, "bf16", 16)
    done = torch.rand(7, 6, generator=gen, device="cuda") < 0.3
    lens = torch.randint(1, 9, (7, 6), generator=gen, device="cuda", dtype=torch.int32)
    want = S.beam_select(x, s, finished=done, lengths=lens, length_penalty=1.0, end_token=3)
    out = {"scores": s, "finished": done, "lengths": lens, "parents": torch.empty_like(lens), "tokens": torch.empty_like(lens)}
    got = S.beam_select(x, s, finished=done, lengths=lens, length_penalty=1.0, end_token=3, out=out)
    assert got is out and all(torch.equal(got[k], want[k]) for k in want)
    with pytest.raises(ValueError):
        S.beam_select(x, s, finished=done, out={"scores": s})
    for n in (65, -1, 2 ** 32 + 3):
        with pytest.raises(S.ShadowKVError):
            S.beam_select(x, s, n_out=n)
    for bad in (dict(end_token=2 ** 32), dict(lengths=lens[:, :5]), dict(lengths=lens.long()), dict(finished=done.int())):
        with pytest.raises(ValueError):
            S.beam_select(x, s, **bad)
    for bad in (x.transpose(1, 2), x.double(), x[0], x[..., ::2]):
        with pytest.raises(ValueError):
            S.beam_select(bad, s)
    assert S.beam_select(x[:0], s[:0])["tokens"].shape == (0, 6)


def test_the_same_call_gives_the_same_bits():
    x, s, _ = draw(3, 8, 60001, "bf16", 17)
    a = S.beam_select(x, s, n_out=32)
    rows = torch.randn(3, 60000 * 8 + 60001 + 7, device="cuda").to(torch.bfloat16)
    odd = rows.as_strided((3, 8, 60001), (rows.shape[1], 60001, 1), 7)   # the same logits at other addresses
    odd.copy_(x)
    for _ in range(3):
        b = S.beam_select(odd, s, n_out=32)
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_another_stream_and_captured_calls():
    x, s, _ = draw(4, 4, 5003, "bf16", 18)
    want = S.beam_select(x, s, n_out=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = S.beam_select(x, s, n_out=8, stream=side)
    side.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = S.beam_select(x, s, n_out=8)
    for seed in range(4):
        new, scores, _ = draw(4, 4, 5003, "bf16", 100 + seed)
        x.copy_(new)
        s.copy_(scores)
        graph.replay()
        torch.cuda.synchronize()
        again = S.beam_select(x, s, n_out=8)
        assert all(torch.equal(out[k], again[k]) for k in out)
        check_choice(out, choose(x, s.cpu(), 8))
