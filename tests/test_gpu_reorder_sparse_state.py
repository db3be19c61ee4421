"""The state of sparse decoding follows its beams: what differs between the rows of a group -- the context behind the prompt, the recent tokens --
reordered in place, against a decode on copies of the parents' whole state."""
import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from workloads import Workload, generate, generated_chunk, with_capacity

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,beams,d,c", [(2, 3, 128, 8), (1, 4, 64, 4), (3, 2, 96, 16)])
def test_decoding_goes_on_from_the_parents_state(groups, beams, d, c):
    rows = groups * beams
    wl = Workload(name="beams", batch=rows, n_q_heads=8, n_kv_heads=2, head_dim=d, ctx_len=64 * c, chunk_size=c, rank=64, n_outlier_chunks=3,
                  topk_chunks=20, local_len=5, rope_theta=5e5, seed=groups + d, n_queries=5)
    s, cap = wl.ctx_len, wl.ctx_len + 4 * c
    t = generate(wl, device="cuda")
    first = torch.arange(rows, device="cuda") // beams * beams
    for name in ("k_rope", "v", "A", "B", "k_local", "v_local"):     # a group is one prompt
        t[name] = t[name][first].contiguous()
    t = with_capacity(t, wl, cap)
    pre = S.build_landmarks(S.Params.from_workload(wl, ctx_capacity=cap), t["k_rope"], t["v"])
    k_local, v_local, n_c, gen = t["k_local"], t["v_local"], s // c - wl.n_outlier_chunks, torch.Generator().manual_seed(d)
    for turn in range(3):
        p = S.Params.from_workload(wl, ctx_len=s + turn * c, ctx_capacity=cap)
        k_pre, k_rope, v = generated_chunk(wl, t, turn)              # each row takes its own tokens
        S.append_chunk(p, k_pre, k_rope, v, t["B"], t["A"], pre["landmarks"], pre["landmark_chunk_ids"], t["v"])
        k_local.copy_(torch.randn(k_local.shape, generator=gen))
        v_local.copy_(torch.randn(v_local.shape, generator=gen))
        # (in a group: a prompt's own arrays, outliers among them, are the same in all its rows)
        parents = (torch.randint(0, beams, (groups, beams), generator=gen) + beams * torch.arange(groups)[:, None]).to(torch.int32).cuda()
        state = [t["A"], t["B"], pre["landmarks"], pre["landmark_chunk_ids"], pre["k_outlier"], pre["v_outlier"], k_local, v_local, t["v"]]
        want = [x[parents.flatten().long()] for x in state]
        S.reorder_rows([t["A"][:, s:], pre["landmarks"][:, :, n_c:], pre["landmark_chunk_ids"][:, :, n_c:], t["v"][:, :, s:], k_local, v_local], parents)
        for x, w, grown in zip(state, want, (1, 0, 2, 2, 0, 0, 0, 0, 2)):
            size = s + (turn + 1) * c if x is t["A"] or x is t["v"] else n_c + turn + 1
            x, w = (x.narrow(grown, 0, size), w.narrow(grown, 0, size)) if grown else (x, w)
            assert torch.equal(x, w)
        # queries near the new chunks, so that these are attended to
        q = (t["q_pool"][turn].float() + 4.0 * k_rope.float()[parents.flatten().long()].mean(2).repeat_interleave(wl.group, 1)).to(torch.bfloat16)
        now = S.Params.from_workload(wl, ctx_len=s + (turn + 1) * c, ctx_capacity=cap)
        out, ids, _ = S.decode_step(now, q, *state, t["pos_offset"])
        out_want, ids_want, _ = S.decode_step(now, q, *want, t["pos_offset"])
        assert torch.equal(ids, ids_want) and torch.equal(out, out_want)
        assert bool((ids == s // c + turn).any(-1).all())            # the chunk that was reordered
