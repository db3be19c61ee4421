"""Measured operators of a prompt's way into the cache: rotary positions, appending to a paged cache, attention of new
tokens over it.

A case is a dict of plain values: the operator (``op``) and its sizes.  ``prepare`` makes what a serving program has in
hand before the call, ``run`` makes the call: with ``own`` through the library's entry points, without it in plain torch
operations (32 bits, 64 for angles, rounded once).  ``exact`` gives the same outputs in 64 bits from the definition.

    rotate   ``rotate``: heads of [seqs, tokens, heads, d] turned to their positions, into [seqs, heads, tokens, d] or the
             same order; the pairs of a head lie half a head apart (``half``) or side by side (``interleaved``)
    append   ``paged_append``: keys (rotated on the way) and values of ragged runs of new tokens into the pages of their
             sequences, their queries rotated beside them
    attend   ``paged_attention``: new tokens of each sequence over its pages, causal

Keys are normal with a deviation of 3, which spreads attention logits by 3; values and queries are normal.
"""
from __future__ import annotations

import math

import torch

own = False

_BASE = {"hq": 32, "hkv": 8, "d": 128, "fp8": False}


def _case(name, op, **kw):
    return {"name": name, "op": op, **_BASE, **kw}


def _rope(**kw):
    out = {"rot": 128, "layout": "half", "scaling": "none", "theta": 5e5, "factor": 1.0, "low": 0.0, "high": 0.0, "orig": 0}
    out.update(kw)
    return out


def listed():
    return [
        # the queries of one decode step of 16 long chats, frequencies scaled in bands: latency is all there is
        _case("rotate-query-16x1", "rotate", b=16, s=1, h=32, at=131072, to_heads=False, transposed=False,
              **_rope(scaling="bands", factor=8.0, low=1.0, high=4.0, orig=8192)),
        # pre-RoPE keys of four prompts as a projection leaves them, into the layout that landmarks are built from
        _case("rotate-keys-4x32k", "rotate", b=4, s=32768, h=8, at=0, to_heads=True, transposed=False, **_rope()),
        # half of heads of 96, pairs side by side, stretched contexts, FP8 storage on both sides, undone (or the gradient)
        _case("rotate-partial-3x20k-fp8", "rotate", b=3, s=20001, h=32, at=70000, to_heads=False, transposed=True,
              **{**_BASE, "hkv": 32, "d": 96, "fp8": True},
              **_rope(rot=48, layout="interleaved", scaling="yarn", theta=1e4, factor=16.0, low=1.0, high=32.0, orig=4096)),
        # one decode step of 64 chats: a token each, at ragged lengths
        _case("append-token-64", "append", b=64, n_lo=1, n_hi=1, len_lo=200, len_hi=1000, page=64, **_rope()),
        # prompts joining: ragged chunks of a 28-head model into an FP8 cache of small pages
        _case("append-chunk-6-fp8", "append", b=6, n_lo=500, n_hi=4000, len_lo=4000, len_hi=6000, page=16,
              **{**_BASE, "hq": 28, "hkv": 4, "fp8": True}, **_rope(scaling="linear", factor=4.0)),
        # a single chat with a short context
        _case("attend-token-1x4k", "attend", b=1, n_lo=1, n_hi=1, len_lo=4000, len_hi=4000, page=16),
        # the ordinary dense decode step: a batch of ragged contexts
        _case("attend-token-16x32k", "attend", b=16, n_lo=1, n_hi=1, len_lo=8000, len_hi=32768, page=64),
        # the longest context, one sequence, sixteen query heads per KV head
        _case("attend-token-1x1m", "attend", b=1, n_lo=1, n_hi=1, len_lo=1048576, len_hi=1048576, page=64, **{**_BASE, "hkv": 2}),
        # a few drafted tokens of 24 chats checked at once (some sequences have none), small heads, seven to a KV head, FP8
        _case("attend-drafts-24-fp8", "attend", b=24, n_lo=0, n_hi=5, len_lo=3000, len_hi=20000, page=32,
              **{**_BASE, "hq": 14, "hkv": 2, "d": 64, "fp8": True}),
        # chunks of prompts beside single tokens, heads of 96 without groups, FP8 cache
        _case("attend-chunk-4x1k-fp8", "attend", b=4, n_lo=1, n_hi=1300, len_lo=5000, len_hi=9000, page=64,
              **{**_BASE, "hkv": 32, "d": 96, "fp8": True}),
        # a chunk of a long prompt over what is already there
        _case("attend-chunk-1x2k-of-30k", "attend", b=1, n_lo=2048, n_hi=2048, len_lo=30011, len_hi=30011, page=64),
        # a whole prompt
        _case("attend-prompt-1x8k", "attend", b=1, n_lo=8192, n_hi=8192, len_lo=8192, len_hi=8192, page=128),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges: any operator, 1 to 64 sequences, runs of one to 8K new tokens, contexts of 64 to 1M
    tokens (no more keys, scores or elements in all than the largest listed case of the operator), the head layouts in use,
    both storage types, pages of 16 to 256 tokens."""
    op = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 2, 128), (64, 8, 128), (32, 32, 96), (16, 8, 64), (14, 2, 64)])
    case = {"op": op, "hq": hq, "hkv": hkv, "d": d, "fp8": rng.random() < 0.4}
    rot = rng.choice([d, d, d // 2, d // 4 // 8 * 8])
    scaling = rng.choice(["none", "none", "linear", "ntk", "bands", "yarn"])
    rope = _rope(rot=rot, layout=rng.choice(["half", "half", "interleaved"]), scaling=scaling, theta=rng.choice([1e4, 5e5]))
    if scaling != "none":
        rope["factor"] = rng.choice([2.0, 4.0, 8.0, 32.0])
    if scaling in ("bands", "yarn"):
        rope.update(orig=rng.choice([4096, 8192]), low=1.0, high=4.0 if scaling == "bands" else 32.0)
    if op == "rotate":
        b, h = _log_uniform(rng, 1, 16), rng.choice([hq, hkv])
        s = _log_uniform(rng, 1, max(2, 2 ** 27 // (b * h * d)))
        case.update(b=b, s=s, h=h, at=rng.choice([0, 1000, 100000, 1000000]), to_heads=rng.random() < 0.5, transposed=rng.random() < 0.3, **rope)
        return case
    if op == "append":
        b = _log_uniform(rng, 1, 64)
        n_hi = 1 if rng.random() < 0.4 else _log_uniform(rng, 1, max(2, 2 ** 26 // (b * hq * d)))
        n_lo = rng.randint(0, 1) if n_hi > 1 else n_hi
        len_hi = n_hi + _log_uniform(rng, 1, max(2, 2 ** 26 // (b * hkv * d)))
        case.update(b=b, n_lo=n_lo, n_hi=n_hi, len_lo=n_hi, len_hi=len_hi, page=rng.choice([16, 32, 64, 128, 256]), **rope)
        return case
    if rng.random() < 0.5:                               # single tokens, or a few
        n_hi = rng.choice([1, 1, 1, 4, 8])
        b = _log_uniform(rng, 1, 64)
        keys = 2 ** 29 // (hkv * d)                      # 2^29 elements of K in all
        keys = min(keys, 1_900_000_000 // (hq * n_hi))
    else:
        b = _log_uniform(rng, 1, 8)
        n_hi = _log_uniform(rng, 16, max(17, 8192 // b))
        keys = min(2 ** 28 // (hkv * d), 1_900_000_000 // (hq * n_hi))   # as many scores
    len_hi = max(n_hi, min(1048576, _log_uniform(rng, 64, max(65, keys // b))))
    case.update(b=b, n_lo=rng.choice([n_hi, rng.randint(0, 1)]) if n_hi > 1 else 1, n_hi=n_hi, len_lo=max(n_hi, len_hi // 4), len_hi=len_hi,
                page=rng.choice([16, 32, 64, 128, 256]))
    return case


# ---- sizes and inputs -------------------------------------------------------------------------------------------------

def _spread(lo, hi, b, turn):
    """b whole numbers of [lo, hi], both ends among them (b = 1: hi), in a fixed shuffled order; no two cases need a seed."""
    if b == 1:
        return [hi]
    return [lo + (hi - lo) * ((turn * i + 1) % b) // (b - 1) if b > 2 else (lo, hi)[i] for i in range(b)]


def _lengths(case):
    """Per sequence: new tokens, and tokens in the cache with them."""
    b = case["b"]
    turn = next(t for t in (7, 5, 3, 11, 13, 17) if b % t)
    return _spread(case["n_lo"], case["n_hi"], b, 1), _spread(case["len_lo"], case["len_hi"], b, turn)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _storage(case):
    return torch.float8_e5m2 if case["fp8"] else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "rotate":
        b, n, h, d = case["b"], case["s"], case["h"], case["d"]
        s["x"] = _randn(gen, b, n, h, d).mul_(3).to(_storage(case))
        s["pos"] = torch.randint(0, 1 + min(case["at"], 4096), (b,), generator=gen, device="cuda", dtype=torch.int32) + max(0, case["at"] - 4096)
        return s
    news, lens = _lengths(case)
    b, hq, hkv, d, ps = case["b"], case["hq"], case["hkv"], case["d"], case["page"]
    width = -(-max(lens) // ps)
    used = [-(-n // ps) for n in lens]
    total = sum(used)
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)      # pages come as they were free
    table = torch.zeros(b, width, dtype=torch.int32)
    places = [(i, j) for i, n in enumerate(used) for j in range(n)]
    at = torch.tensor(places, dtype=torch.int64).t().cuda()
    s["table"] = table.cuda().index_put_((at[0], at[1]), order)
    s["k_cache"] = _randn(gen, total, hkv, ps, d).mul_(3).to(_storage(case))
    s["v_cache"] = _randn(gen, total, hkv, ps, d).to(_storage(case))
    starts = torch.tensor([sum(news[:i]) for i in range(b + 1)], dtype=torch.int32)
    s["starts"], s["lens"] = starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    t = sum(news)
    s["tokens"], s["most_new"], s["most"] = t, max(news), max(lens)
    s["q"] = _randn(gen, t, hq, d)
    if case["op"] == "append":
        s["k"], s["v"] = _randn(gen, t, hkv, d).mul_(3), _randn(gen, t, hkv, d)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _own_rope(S, case):
    scaling = {"none": S.ROPE_PLAIN, "linear": S.ROPE_LINEAR, "ntk": S.ROPE_NTK, "bands": S.ROPE_BANDS, "yarn": S.ROPE_YARN}[case["scaling"]]
    return S.Rope(head_dim=case["d"], rot_dim=case["rot"], layout=S.ROPE_HALF if case["layout"] == "half" else S.ROPE_INTERLEAVED,
                  scaling=scaling, theta=case["theta"], factor=case["factor"], low=case["low"], high=case["high"], original_len=case["orig"])


def _frequencies(case):
    """Radians per position of each pair, in 64 bits, and what cosine and sine are multiplied by."""
    rot, f = case["rot"], case["factor"]
    base = case["theta"] * (f ** (rot / (rot - 2)) if case["scaling"] == "ntk" else 1.0)
    w = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if case["scaling"] == "linear":
        return w / f, 1.0
    if case["scaling"] == "bands":                      # by the turns a pair makes in the original length
        keep = ((case["orig"] * w / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])).clamp(0, 1)
        return w * keep + w / f * (1 - keep), 1.0
    if case["scaling"] == "yarn":                       # by the pair's index, between those that make high and low turns
        at = lambda turns: rot * math.log(case["orig"] / (turns * 2 * math.pi)) / (2 * math.log(case["theta"]))  # noqa: E731
        first, last = max(math.floor(at(case["high"])), 0), min(math.ceil(at(case["low"])), rot - 1)
        gone = ((torch.arange(rot // 2, dtype=torch.float64, device="cuda") - first) / max(last - first, 1e-3)).clamp(0, 1)
        return w / f * gone + w * (1 - gone), 0.1 * math.log(f) + 1.0
    return w, 1.0


def _turned(case, x, pos, transposed=False):
    """x [..., h, d] in 32 bits, pos [...]: rotated."""
    w, m = _frequencies(case)
    rot, half = case["rot"], case["rot"] // 2
    a = pos.to(torch.float64)[..., None, None] * w
    c, s = (a.cos() * m).float(), (a.sin() * m).float()
    if transposed:
        s = -s
    y = x.clone()
    if case["layout"] == "half":
        p, q = x[..., :half], x[..., half:rot]
        y[..., :half], y[..., half:rot] = p * c - q * s, q * c + p * s
    else:
        p, q = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = p * c - q * s, q * c + p * s
    return y


def _where(s):
    """Sequence of every new token, and its place in the cache."""
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    place = s["lens"].long()[seq] - (s["starts"][1:].long()[seq] - t)
    return seq, place


def _plain_rotate(s):
    case, x = s["case"], s["x"]
    pos = s["pos"][:, None] + torch.arange(case["s"], device="cuda")
    y = _turned(case, x.float(), pos, case["transposed"]).to(x.dtype)
    return y.transpose(1, 2).contiguous() if case["to_heads"] else y


def _plain_append(s):
    case, ps = s["case"], s["case"]["page"]
    seq, place = _where(s)
    page, row = s["table"][seq, place // ps].long(), place % ps
    s["k_cache"][page, :, row] = _turned(case, s["k"].float(), place).to(s["k_cache"].dtype)
    s["v_cache"][page, :, row] = s["v"].to(s["v_cache"].dtype)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": _turned(case, s["q"].float(), place).to(torch.bfloat16)}


def _plain_attend(s):
    case = s["case"]
    b, hq, hkv, d = case["b"], case["hq"], case["hkv"], case["d"]
    n, most = s["most_new"], s["most"]

    def dense(cache):                                   # [pages, hkv, ps, d] -> [b, hkv, length, d]
        x = cache[s["table"].long()]
        return x.transpose(1, 2).reshape(b, hkv, -1, d)[:, :, :most].float()

    seq, place = _where(s)
    local = torch.arange(s["tokens"], device="cuda") - s["starts"].long()[seq]
    q = torch.zeros(b, n, hq, d, device="cuda")
    last = torch.full((b, n), -1, dtype=torch.int64, device="cuda")
    q[seq, local], last[seq, local] = s["q"].float(), place
    q = q.view(b, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    p = torch.matmul(q, dense(s["k_cache"]).transpose(2, 3)).mul_(1 / math.sqrt(d)).view(b, hkv, hq // hkv, n, most)
    p.masked_fill_((torch.arange(most, device="cuda") > last[..., None])[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True).clamp_(min=1e-30)
    o = torch.matmul(p.view(b, hkv, -1, most), dense(s["v_cache"])).view(b, hkv, -1, n, d) / total
    return o.permute(0, 3, 1, 2, 4).reshape(b, n, hq, d)[seq, local].to(torch.bfloat16)


def run(state):
    s, case = state, state["case"]
    if not own:
        return _plain_rotate(s) if case["op"] == "rotate" else _plain_append(s) if case["op"] == "append" else _plain_attend(s)
    from paper_2410_21465_amd import shadowkv as S
    if case["op"] == "rotate":
        out = torch.empty(case["b"], case["h"], case["s"], case["d"], dtype=s["x"].dtype, device="cuda").transpose(1, 2) if case["to_heads"] else None
        y = S.rotate(_own_rope(S, case), s["x"], out=out, pos_offset=s["pos"], transposed=case["transposed"])
        return y.transpose(1, 2) if case["to_heads"] else y
    cache = S.PagedCache(s["k_cache"], s["v_cache"], s["table"])
    if case["op"] == "append":
        q = S.paged_append(cache, s["k"], s["v"], s["lens"], seq_starts=s["starts"], rope=_own_rope(S, case), q=s["q"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": q}
    return S.paged_attention(cache, s["q"], s["lens"], seq_starts=s["starts"])


def work(case):
    eb, d = 1 if case["fp8"] else 2, case["d"]
    if case["op"] == "rotate":
        n = case["b"] * case["s"] * case["h"]
        return {"bytes": 2 * n * d * eb, "flops": 3 * n * case["rot"]}
    news, lens = _lengths(case)
    t = sum(news)
    if case["op"] == "append":
        return {"bytes": t * d * (4 * case["hq"] + case["hkv"] * (4 + 2 * eb)), "flops": 3 * t * case["rot"] * (case["hq"] + case["hkv"])}
    seen = sum(n * m - n * (n - 1) // 2 for n, m in zip(news, lens))          # keys that tokens attend over
    keys = sum(m for n, m in zip(news, lens) if n)
    return {"bytes": 4 * t * case["hq"] * d + 2 * keys * case["hkv"] * d * eb, "flops": 4 * seen * case["hq"] * d}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    def spun(x, pos, sign=1.0):
        """x [n, h, d] in 64 bits at positions pos [n]: every pair a complex number times m e^(i a)."""
        rot, f, pairs = case["rot"], case["factor"], case["rot"] // 2
        speed, m = [], 1.0
        for p in range(pairs):
            w = case["theta"] ** (-2.0 * p / rot)
            if case["scaling"] == "ntk":
                w = (case["theta"] * f ** (rot / (rot - 2.0))) ** (-2.0 * p / rot)
            elif case["scaling"] == "linear":
                w /= f
            elif case["scaling"] == "bands":
                length = 2 * math.pi / w
                if length > case["orig"] / case["low"]:
                    w /= f
                elif length >= case["orig"] / case["high"]:
                    g = (case["orig"] / length - case["low"]) / (case["high"] - case["low"])
                    w = (1 - g) * w / f + g * w
            elif case["scaling"] == "yarn":
                ends = [rot * math.log(case["orig"] / (2 * math.pi * turns)) / (2 * math.log(case["theta"])) for turns in (case["high"], case["low"])]
                lo, hi = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), rot - 1)
                g = min(1.0, max(0.0, (p - lo) / max(hi - lo, 1e-3)))
                w, m = g * w / f + (1 - g) * w, 0.1 * math.log(f) + 1.0
            speed.append(w)
        a = pos.double()[:, None, None] * torch.tensor(speed, dtype=torch.float64, device=x.device)
        unit = torch.polar(torch.full_like(a, m), sign * a)
        head = x[..., :rot]
        z = torch.complex(head[..., :pairs], head[..., pairs:]) if case["layout"] == "half" else torch.view_as_complex(head.reshape(*head.shape[:-1], pairs, 2).contiguous())
        z = z * unit
        y = torch.cat([z.real, z.imag], -1) if case["layout"] == "half" else torch.view_as_real(z).reshape(head.shape)
        return torch.cat([y, x[..., rot:]], -1)

    s = prepare(case, seed)
    if case["op"] == "rotate":
        rows = []
        for i in range(case["b"]):
            pos = int(s["pos"][i]) + torch.arange(case["s"], device="cuda")
            rows.append(spun(s["x"][i].double(), pos, -1.0 if case["transposed"] else 1.0))
        y = torch.stack(rows)
        return y.transpose(1, 2).contiguous() if case["to_heads"] else y
    news, lens = _lengths(case)
    table, ps, d, hkv = s["table"].tolist(), case["page"], case["d"], case["hkv"]
    if case["op"] == "append":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for i, (n, m) in enumerate(zip(news, lens)):
            if not n:
                continue
            place = torch.arange(m - n, m, device="cuda")
            page, row = torch.tensor(table[i], device="cuda")[place // ps], place % ps
            kc[page, :, row] = spun(s["k"][at:at + n].double(), place)
            vc[page, :, row] = s["v"][at:at + n].double()
            q[at:at + n] = spun(s["q"][at:at + n].double(), place)
            at += n
        return {"k_cache": kc, "v_cache": vc, "q": q}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, at = case["hq"] // hkv, 0
    for i, (n, m) in enumerate(zip(news, lens)):
        pages = torch.tensor(table[i][:-(-m // ps)], device="cuda")
        for h in range(hkv if n else 0):
            k = s["k_cache"][pages, h].reshape(-1, d)[:m].double()
            v = s["v_cache"][pages, h].reshape(-1, d)[:m].double()
            for g in range(h * group, (h + 1) * group):
                for j in range(0, n, 2048):              # 2048 tokens at a time: the scores in 64 bits
                    x = s["q"][at + j:at + min(n, j + 2048), g].double()
                    w = x @ k.t() / math.sqrt(d)
                    see = torch.arange(m, device="cuda")[None] <= (m - n + j + torch.arange(len(x), device="cuda"))[:, None]
                    out[at + j:at + j + len(x), g] = torch.softmax(w.masked_fill(~see, -math.inf), -1) @ v
        at += n
    return out
