"""Where the paged operators and the sparse decode step meet: a prompt appended through pages, and rotations far along a context."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import BF, attention, check_turned, pair_size, turned

pytestmark = pytest.mark.gpu


def _q(n, hq, d, seed):
    return torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


def test_a_decode_step_over_an_appended_prompt_attends_over_its_keys():
    """A prompt appended to dense arrays through their pages, then build_landmarks, factorize_keys and a decode step whose budget covers
    everything.  Its output is that of attention in 64 bits over the keys that it is given: the stored ones of the outlier chunks, and A B
    rotated elsewhere.  Queries are large enough that a few keys hold most of a row's weight.

    Tolerances: a rounding to bf16 (2^-8); weights in two bf16 terms and the exponentials (2^-16 + 2^-20); twice the error of the logits, made
    of the rebuilt keys' -- r + 4 fp32 steps of the sum |A| |B| and the 2^-19 of a pair that a rotation may be off by -- and of d + 16 fp32
    steps of the products' sum.  Chunks left out, keys not rotated, or rotated one position on, are out of them."""
    b, hq, hkv, d, s, r, c, o = 2, 8, 2, 64, 512, 40, 8, 4
    gen = torch.Generator(device="cuda").manual_seed(4)
    low = torch.randn(b, s, 32, generator=gen, device="cuda") @ torch.randn(32, hkv * d, generator=gen, device="cuda") / 6
    k_pre, v = low.to(BF), torch.randn(b, s, hkv * d, generator=gen, device="cuda").to(BF)
    k_rope, store = (torch.empty(b, hkv, s, d, dtype=BF, device="cuda") for _ in range(2))
    cache = S.dense_pages(k_rope, store, 64)
    rope = S.Rope(d, theta=5e5)
    lens = torch.full((b,), s, dtype=torch.int32, device="cuda")
    S.paged_append(cache, k_pre.view(b * s, hkv, d), v.view(b * s, hkv, d), lens, rope=rope)
    p = S.Params(b, hq, hkv, d, s, chunk_size=c, rank=r, n_outlier_chunks=o, topk_chunks=s // c - o, local_len=0)
    pre, fac = S.build_landmarks(p, k_rope, store), S.factorize_keys(p, k_pre)
    q = (_q(b, hq, d, 5).float() * 4).to(BF)
    out, _, _ = S.decode_step(p, q, fac["A"], fac["B"], pre["landmarks"], pre["landmark_chunk_ids"], pre["k_outlier"],
                              pre["v_outlier"], None, None, store)
    # everything else on the CPU in 64 bits
    q, out, A, B, k_rope, store, ids = (x.cpu() for x in (q.double(), out.double(), fac["A"].double(), fac["B"].double(), k_rope.double(),
                                                          store.double(), pre["outlier_chunk_ids"]))
    pos, last = torch.arange(s), torch.tensor([s - 1])
    for i in range(b):
        raw = torch.stack([A[i] @ B[i, h] for h in range(hkv)], 1)                                  # [s, hkv, d]
        size = torch.stack([A[i].abs() @ B[i, h].abs() for h in range(hkv)], 1)
        stored = torch.zeros(s, hkv, dtype=torch.bool)
        for h in range(hkv):
            for chunk in ids[i, h].tolist():
                stored[chunk * c:(chunk + 1) * c, h] = True

        def result(keys, see=None):
            keys = torch.where(stored[..., None], k_rope[i].transpose(0, 1), keys)
            return keys, attention(q[i:i + 1], keys, store[i].transpose(0, 1), last, d ** -0.5, see)

        keys, (want, _, av, qk) = result(turned(rope, raw, pos))
        key_err = torch.where(stored[..., None], torch.zeros(()).double(), (r + 4) * 2.0 ** -24 * 2 * pair_size(rope, size) + 2.0 ** -19 * pair_size(rope, raw))
        logit = torch.stack([(q[i, g].abs() * key_err[:, g // (hq // hkv)]).sum(-1).amax() * d ** -0.5 for g in range(hq)])
        delta = 2 * (logit + (d + 16) * 2.0 ** -24 * qk[0])[None, :, None]
        tol = 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (2.0 ** -16 + 2.0 ** -20 + delta) * av
        err = (out[i:i + 1] - want).abs()
        assert (err <= tol).all(), f"sequence {i}: {(err - tol).max().item()} over"
        # what the tolerance has to tell apart
        gone = torch.zeros(s, dtype=torch.bool)
        gone[200:232] = True
        for wrong in (result(turned(rope, raw, pos), gone), result(raw), result(turned(rope, raw, pos + 1))):
            assert ((out[i:i + 1] - wrong[1][0]).abs() > tol).float().mean() > 0.5
        # and the rebuilt keys are the appended ones, to what the factors leave out and round (2^-8 each of |A| |B|, 2^-8 of the key): by norm
        tail = torch.linalg.svdvals(k_pre[i].double().cpu())[r:].norm()
        off = (turned(rope, raw, pos) - k_rope[i].transpose(0, 1)).norm()
        assert off <= 1.1 * tail + 2.0 ** -7 * size.norm() + 2.0 ** -8 * k_rope[i].norm()
        assert off < 0.1 * (raw - k_rope[i].transpose(0, 1)).norm()


@pytest.mark.parametrize("at", [0, 131072, 1048576 - 512])
def test_rotations_far_along_agree_where_both_get_the_same_frequencies(at):
    """A decode step takes its frequencies in fp32.  Keys that it rebuilds are those that `rotate` makes with the same fp32 numbers as its
    inv_freq, wherever they stand; with the unrounded ones they are up to 2^-25 of the position in radians apart."""
    b, hkv, d, s, r = 1, 2, 64, 512, 64
    scaled = S.Rope(d, scaling=S.ROPE_BANDS, factor=8.0, low=1.0, high=4.0, original_len=8192)
    inv = scaled.frequencies().float().cuda()
    gen = torch.Generator(device="cuda").manual_seed(8)
    rows = torch.randn(hkv, r, d, generator=gen, device="cuda").to(BF)
    A = torch.eye(r, device="cuda").repeat(s // r, 1)[None].to(BF).contiguous()                     # token t is row t % r of B, exactly
    keys = rows.transpose(0, 1).repeat(s // r, 1, 1)                                                # [s, hkv, d]
    p = S.Params(b, 4, hkv, d, s, chunk_size=8, rank=r, n_outlier_chunks=0, topk_chunks=s // 8, local_len=0, inv_freq=inv,
                 flags=S.FLAG_KEEP_REBUILT_KEYS)
    off = torch.tensor([at], dtype=torch.int32, device="cuda")
    k_rope = S.rotate(S.Rope(d, inv_freq=inv), keys[None], pos_offset=off)
    store = torch.randn(b, hkv, s, d, generator=gen, device="cuda").to(BF)
    pre = S.build_landmarks(p, k_rope.transpose(1, 2).contiguous(), store)
    _, ids, ws = S.decode_step(p, _q(b, 4, d, 9), A, rows[None].contiguous(), pre["landmarks"], pre["landmark_chunk_ids"], pre["k_outlier"],
                               pre["v_outlier"], None, None, store, off)
    assert torch.equal(ids[0], torch.arange(s // 8, dtype=torch.int32, device="cuda").expand(hkv, -1))
    rebuilt = S.workspace_view(p, ws, "k_sparse")[0].transpose(0, 1).double()                       # [s, hkv, d], fp32
    pos = at + torch.arange(s, device="cuda")
    check_turned(S.Rope(d), k_rope[0], keys, pos, freq=inv.double().cpu())
    size = pair_size(S.Rope(d), keys.double())
    assert ((rebuilt - k_rope[0].double()).abs() <= 2.0 ** -8 * rebuilt.abs() + 2.0 ** -18 * size).all()
    apart = (turned(S.Rope(d), keys.double(), pos, freq=scaled.frequencies()) - rebuilt).abs() / size
    assert (apart <= 2.0 ** -25 * (at + s) + 2.0 ** -18).all()
    if at > 1000000:
        assert apart.max() > 2.0 ** -8                                                              # more than a rounding to bf16
