"""A beam search over the paged cache as a serving program makes it -- choice, pages and dense state that follow it, append, attention --
against the same search that keeps every beam's whole history in dense 64-bit arrays."""
import math

import pytest
import torch

from paper_2410_21465_amd import shadowkv as S
from paged_util import attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,beams,page,fp8", [(3, 4, 16, False), (2, 5, 8, True), (1, 1, 64, False)])
def test_beam_search_over_pages(groups, beams, page, fp8):
    gen = torch.Generator(device="cuda").manual_seed(groups * beams)
    hq, hkv, d, vocab, layers, steps, end = 4, 2, 64, 301, 2, 14, 7
    rows, dtype = groups * beams, torch.float8_e5m2 if fp8 else torch.bfloat16
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    embed = [(rand(vocab, hq + 2 * hkv, d) * 1.5).to(torch.bfloat16) for _ in range(layers)]      # a token's q, k, v in each layer
    head = rand(layers * hq * d, vocab) / math.sqrt(layers * hq * d) * 4
    rope = S.Rope(head_dim=d, theta=1e4)
    prompts = [torch.randint(0, vocab, (n,), generator=gen, device="cuda") for n in (37, 16, 5)[:groups]]

    width = 8 * (64 // page)
    pool = S.PagePool(rows, width, rows * width, page)
    caches = [pool.cache(*(rand(rows * width, hkv, page, d).to(dtype) for _ in "kv")) for _ in range(layers)]

    def forward(tokens, starts=None):
        """New tokens of the rows that have some through all layers: attention outputs [tokens, layers * hq * d]."""
        outs = []
        for l, c in enumerate(caches):
            x = embed[l][tokens]
            q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
            q = S.paged_append(c, k, v, pool.kv_lens, seq_starts=starts, rope=rope, q=q)
            outs.append(S.paged_attention(c, q, pool.kv_lens, seq_starts=starts))
        return torch.cat(outs, 1).flatten(1)

    def dense(history):
        """The same for the last token of one history, in 64 bits, from keys as the cache stores them."""
        outs = []
        for l in range(layers):
            x = embed[l][history]
            turned = S.rotate(rope, x[None, :, :hq + hkv].contiguous())[0]
            q, k, v = turned[-1:, :hq].double(), turned[:, hq:].to(dtype), x[:, hq + hkv:].to(dtype)
            if fp8:
                k = S.rotate(rope, x[None, :, hq:hq + hkv].contiguous(), out=torch.empty(1, len(history), hkv, d, dtype=dtype, device="cuda"))[0]
            outs.append(attention(q, k.double(), v.double(), torch.tensor([len(history) - 1], device="cuda"), 1 / math.sqrt(d))[0])
        return torch.cat(outs, 1).flatten()

    # the prompts go to the first beam of each group
    lens = [len(prompts[i // beams]) if i % beams == 0 else 0 for i in range(rows)]
    pool.update(n_new=torch.tensor(lens, dtype=torch.int32, device="cuda"), caches=caches)
    starts = torch.tensor([sum(lens[:i]) for i in range(rows + 1)], dtype=torch.int32, device="cuda")
    hidden = forward(torch.cat(prompts), starts)[starts[1:].long() - 1]
    scores = torch.full((groups, beams), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    finished = torch.zeros(groups, beams, dtype=torch.bool, device="cuda")
    lengths = torch.zeros(groups, beams, dtype=torch.int32, device="cuda")
    tokens_so_far = torch.full((rows, steps), -1, dtype=torch.int32, device="cuda")
    recent = torch.zeros(rows, layers * hq * d, dtype=torch.float32, device="cuda")       # dense state: last outputs of every row
    recent[::beams] = hidden[::beams].float()
    histories = [prompts[i // beams].tolist() if i % beams == 0 else None for i in range(rows)]
    for step in range(steps):
        logits = (recent @ head).view(groups, beams, vocab)
        best = S.beam_select(logits, scores, finished=finished, lengths=lengths, length_penalty=0.7, end_token=end,
                             out={"scores": scores, "finished": finished, "lengths": lengths,
                                  "parents": torch.empty(groups, beams, dtype=torch.int32, device="cuda"),
                                  "tokens": torch.empty(groups, beams, dtype=torch.int32, device="cuda")})
        parents, chosen = best["parents"].reshape(-1), best["tokens"].reshape(-1)
        S.reorder_rows([tokens_so_far, recent], parents)
        tokens_so_far[:, step] = chosen
        grows = ((parents >= 0) & ~finished.reshape(-1)).int()
        pool.update(parents=parents, n_new=grows, caches=caches)
        if step % 3 == 1:
            pool.compact(caches=caches)
        # histories of every row, as a plain search keeps them
        p, t, g = parents.tolist(), chosen.tolist(), grows.tolist()
        histories = [None if p[i] < 0 else histories[p[i]] + ([t[i]] if g[i] else []) for i in range(rows)]
        assert pool.kv_lens.tolist() == [0 if h is None else len(h) for h in histories]
        live = [i for i in range(rows) if g[i]]
        if not live:
            break
        starts = torch.tensor([sum(g[:i]) for i in range(rows + 1)], dtype=torch.int32, device="cuda")
        out = forward(chosen[live].long(), starts)
        recent[live] = out.float()
        for i in live:
            want = dense(torch.tensor(histories[i], device="cuda"))
            # one rounding to bf16; weights of two bf16 terms (2^-16); logits of sums of 64 products in fp32, 2 (64 + 16) 2^-24 of up to
            # 100: 2^-10 of values below 8
            assert (out[live.index(i)].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + (2.0 ** -10 + 2.0 ** -16) * 8
        assert bool((tokens_so_far[live, :step + 1] >= 0).all())
    used = torch.zeros(rows * width, dtype=torch.int32, device="cuda")
    held = pool.page_table[pool.page_table >= 0].long()
    used.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    assert torch.equal(used, pool.page_refs)
    pool.update(parents=torch.full((rows,), -1, dtype=torch.int32, device="cuda"))
    assert int(pool.page_refs.abs().sum()) == 0 and int(pool.kv_lens.sum()) == 0
