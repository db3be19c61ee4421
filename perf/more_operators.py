"""Measured operators of a search over several continuations: the choice over beams and vocabulary, and the state that follows
it, dense or in pages.

A case is a dict of plain values: the operator (``op``) and its sizes.  ``prepare`` makes what a serving program has in
hand before the call, ``run`` makes the call: with ``own`` through the library's entry points, without it in plain torch
operations.  ``exact`` gives the chosen scores in 64 bits from the definition (the other operators move data and compute no numbers).

    select   ``beam_select``: the best continuations of every group of beams, by summed log-probability (over a power of the
             length), ties to the lower beam and token
    reorder  ``reorder_rows``: rows of dense state arrays replaced in place by those of their parents
    update   ``PagePool.update``: sequences in pages become continuations of others (forked, freed, cut, grown), with the copies of
             shared last pages that are about to be written, in every layer
    copy     ``pages_copy``: whole pages to other places, in every layer
    compact  ``PagePool``: sequences leave, the pages of the others move to the lowest places, in every layer, new ones join
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "fp8": torch.float8_e5m2}


def _select(name, **kw):
    return {"name": name, "op": "select", "finished": False, "penalty": 0.0, "first": False, **kw}


def _pages(name, op, **kw):
    return {"name": name, "op": op, "hkv": 8, "d": 128, "dtype": "bf16", **kw}


def listed():
    return [
        # one prompt searched with four beams, a small vocabulary in full precision: latency is all there is
        _select("select-1x4x32k-fp32", groups=1, beams=4, vocab=32000, n=4, dtype="fp32"),
        # the ordinary step: a batch of prompts, twice as many candidates as beams so that ended ones can be set aside
        _select("select-16x4x128k", groups=16, beams=4, vocab=128256, n=8, dtype="bf16"),
        # an odd vocabulary (rows begin at any address), some beams ended, ranked by length-normalised score
        _select("select-24x8x50k-fp16", groups=24, beams=8, vocab=50257, n=8, dtype="fp16", finished=True, penalty=0.8),
        # a wide search of many prompts over a large vocabulary
        _select("select-32x16x256k", groups=32, beams=16, vocab=262144, n=32, dtype="bf16"),
        # what a step of sparse decoding keeps per sequence besides its context: recent keys and values of eight layers, the tokens so far
        {"name": "reorder-recent-16x4", "op": "reorder", "groups": 16, "beams": 4, "moved": 2, "layers": 8, "inner": 8 * 32 * 128, "tokens": 515, "skip": 0},
        # low-rank keys of long sequences, the part behind a shared prompt; rows change in cycles as well
        {"name": "reorder-lowrank-8x4", "op": "reorder", "groups": 8, "beams": 4, "moved": 3, "layers": 2, "inner": 32768 * 160, "tokens": 32769, "skip": 2048 * 160},
        # a step of 16 searches with four beams over prompts in shared pages
        _pages("update-beams-16x4", "update", groups=16, beams=4, moved=2, shared=4000, own_lo=3, own_hi=200, cut=1, n_new=1, page=64, layers=8, gone=0),
        # drafted tokens of 256 chats, most of them rejected, some chats over; small pages in FP8, a prefix that all of a group share
        _pages("update-drafts-64x4-fp8", "update", groups=64, beams=4, moved=1, shared=1000, own_lo=100, own_hi=3001, cut=5, n_new=8, page=16, layers=4,
               gone=1, **{"hkv": 4, "dtype": "fp8"}),
        # a few pages of one layer
        _pages("copy-6", "copy", pairs=6, pages=64, page=16, layers=1),
        # a long prefix given a second home, in all of eight layers
        _pages("copy-500x8", "copy", pairs=500, pages=1024, page=64, layers=8),
        # a pool of short chats of which half leave
        _pages("compact-64-fp8", "compact", rows=64, len_lo=100, len_hi=700, page=16, layers=2, **{"hkv": 2, "d": 64, "dtype": "fp8"}),
        # a large pool of long sequences of which half leave, eight layers
        _pages("compact-32x8k", "compact", rows=32, len_lo=2000, len_hi=8191, page=64, layers=4),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges: any operator; 1 to 64 groups of 1 to 32 beams, vocabularies of 500 to 262144, up to 64
    places; up to 256 sequences of 16 to 16K tokens in pages of 8 to 256, heads in use by the other operators, both storage types.
    No more elements in all than the largest listed case of the operator."""
    op = rng.choice(["select", "select", "select", "reorder", "update", "update", "copy", "compact"])
    if op == "select":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 10, 16, 32])
        groups = _log_uniform(rng, 1, 64)
        n, dtype = min(64, rng.choice([beams, beams, 2 * beams, 2 * beams + 1])), rng.choice(["bf16", "bf16", "fp16", "fp32"])
        most = 2 ** 26 if n > 32 or dtype == "fp32" else 2 ** 27
        case = _select(None, groups=groups, beams=beams, vocab=_log_uniform(rng, 500, min(262144, most // (beams * groups))), n=n, dtype=dtype)
        if rng.random() < 0.3:
            case.update(finished=True, penalty=rng.choice([0.0, 0.6, 1.0]))
        elif rng.random() < 0.2:
            case["first"] = True
        del case["name"]
        return case
    groups, beams = rng.choice([(1, 4), (3, 5), (16, 4), (8, 8), (32, 4), (64, 4), (10, 3), (2, 32)])
    moved = rng.randint(0, beams - 1)
    if op == "reorder":
        inner = 8 * _log_uniform(rng, 64, 2 ** 26 // (groups * beams))
        return {"op": op, "groups": groups, "beams": beams, "moved": moved, "layers": rng.randint(1, 2), "inner": inner,
                "tokens": _log_uniform(rng, 3, 40000), "skip": rng.choice([0, 0, inner // 16 * 8])}
    hkv, d = rng.choice([(8, 128), (4, 128), (2, 128), (8, 64), (2, 64), (4, 96)])
    base = {"op": op, "hkv": hkv, "d": d, "dtype": rng.choice(["bf16", "bf16", "fp8"]), "page": rng.choice([8, 16, 32, 64, 128, 256])}
    room = 2 ** 28 // (hkv * d)                              # tokens of a layer's keys, in all layers together
    if op == "copy":
        layers = rng.randint(1, 8)
        pairs = _log_uniform(rng, 1, max(2, min(4000, room // (2 * layers * base["page"]))))
        return {**base, "pairs": pairs, "pages": 2 * pairs + rng.randint(0, 7), "layers": layers}
    layers = rng.randint(1, 4)
    if op == "update":
        own_hi = _log_uniform(rng, 16, max(17, min(8000, room // (2 * layers * groups * beams))))
        shared = rng.choice([0, _log_uniform(rng, 8, max(9, min(16000, room // (2 * layers * groups))))])
        return {**base, "groups": groups, "beams": beams, "moved": moved, "shared": shared, "own_lo": 8, "own_hi": own_hi, "cut": rng.choice([0, 1, 5]),
                "n_new": rng.choice([1, 1, 1, 4, 40]), "layers": layers, "gone": rng.randint(0, 1) if beams > moved + 1 else 0}
    rows = _log_uniform(rng, 2, 256)
    len_hi = _log_uniform(rng, 16, max(17, min(16000, room // (layers * rows))))
    return {**base, "rows": rows, "len_lo": max(1, len_hi // 8), "len_hi": len_hi, "layers": layers}


# ---- sizes and inputs -------------------------------------------------------------------------------------------------

def _spread(lo, hi, b):
    """b whole numbers of [lo, hi], both ends among them (b = 1: hi), in a fixed shuffled order; no two cases need a seed."""
    if b == 1:
        return [hi]
    turn = next(t for t in (7, 5, 3, 11, 13, 17, 19, 23) if b % t)
    return [lo + (hi - lo) * ((turn * i + 1) % b) // (b - 1) for i in range(b)]


def _parents(case):
    """Row that every row continues: in each group ``moved`` beams give way to lower ones (one of them taken twice, the others shifted by
    one place, in every second group in a cycle), ``gone`` ones end (-1)."""
    out, beams, moved, gone = [], case["beams"], case["moved"], case.get("gone", 0)
    for g in range(case["groups"]):
        p = list(range(beams))
        if moved:
            last = beams - gone
            p[last - moved:last] = range(last - moved - 1, last - 1)
            if g % 2 and moved > 1:
                p[last - moved] = last - 1                     # the rows that moved are a cycle
        for i in range(gone):
            p[beams - 1 - i] = -1
        out += [-1 if x < 0 else g * beams + x for x in p]
    return out


def _beam_lengths(case):
    """update: tokens of every row before the call, what is kept of them, and after it."""
    lens = [case["shared"] + x for x in _spread(case["own_lo"], case["own_hi"], case["groups"] * case["beams"])]
    keep = [n - case["cut"] for n in lens]
    parents = _parents(case)
    after = [0 if p < 0 else keep[p] for p in parents]
    return lens, parents, after, [0 if p < 0 else n + case["n_new"] for n, p in zip(after, parents)]


def _update_pages(case):
    """update: pages of a group's shared prefix, places of a row, pages of the pool."""
    ps, lens = case["page"], _beam_lengths(case)[0]
    prefix = case["shared"] // ps
    width = -(-(max(lens) + case["n_new"]) // ps) + 1
    used = case["groups"] * prefix + sum(-(-n // ps) - prefix for n in lens)
    grown = 2 * len(lens) * (2 + case["n_new"] // ps)
    return prefix, width, used + grown + 5


def _randn(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16).to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _layers(case, gen, n_pages):
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    return [tuple(_randn(gen, *shape, dtype=_TYPES[case["dtype"]]) for _ in "kv") for _ in range(case["layers"])]


def _pool(state, case, width, n_pages, rows):
    """The bookkeeping of a pool and, with ``own``, the library's handle on it, which a program keeps."""
    if own:
        from paper_2410_21465_amd import shadowkv as S
        pool = S.PagePool(rows, width, n_pages, case["page"])
        state["pool"], state["table"], state["lens"], state["refs"] = pool, pool.page_table, pool.kv_lens, pool.page_refs
        state["caches"] = [pool.cache(k, v) for k, v in state["layers"]]
    else:
        state["table"] = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        state["lens"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        state["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda")


def _fill(state, table, lens, order):
    """Page numbers of ``table`` (negative: none) taken through ``order``; lengths; references counted."""
    t = torch.tensor(table, dtype=torch.int64)
    t = torch.where(t >= 0, order.cpu()[t.clamp(min=0)], -1)
    state["table"].copy_(t.to(torch.int32))
    state["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
    state["refs"].copy_(torch.bincount(t[t >= 0], minlength=len(state["refs"])).to(torch.int32))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "select":
        g, b, v = case["groups"], case["beams"], case["vocab"]
        # a language model's logits: a broad bulk, and a few tokens of each row that stand out
        x = torch.randn(g, b, v, generator=gen, device="cuda", dtype=torch.float32).mul_(2.0)
        best = torch.randint(0, v, (g, b, 12), generator=gen, device="cuda")
        x.scatter_add_(2, best, 3.0 + 6.0 * torch.rand(g, b, 12, generator=gen, device="cuda"))
        s["logits"] = x.to(_TYPES[case["dtype"]])
        s["scores"] = -5.0 - 4.0 * torch.rand(g, b, generator=gen, device="cuda")
        if case["first"]:                                      # all beams are the prompt: one of them counts
            s["scores"].fill_(-math.inf)[:, 0] = 0.0
        s["finished"] = torch.rand(g, b, generator=gen, device="cuda") < 0.3 if case["finished"] else None
        s["lengths"] = torch.randint(3, 60, (g, b), generator=gen, device="cuda", dtype=torch.int32) if case["penalty"] else None
        return s
    if case["op"] == "reorder":
        rows = case["groups"] * case["beams"]
        s["parents"] = _ints(_parents(case))
        s["state"] = [_randn(gen, rows, case["inner"]) for _ in range(2 * case["layers"])]
        s["history"] = torch.randint(0, 100000, (rows, case["tokens"]), generator=gen, device="cuda", dtype=torch.int32)
        return s
    if case["op"] == "copy":
        s["layers"] = _layers(case, gen, case["pages"])
        order = torch.randperm(case["pages"], generator=gen, device="cuda").to(torch.int32)
        s["src"], s["dst"] = order[:case["pairs"]].contiguous(), order[case["pairs"]:2 * case["pairs"]].contiguous()
        if own:
            from paper_2410_21465_amd import shadowkv as S
            s["caches"] = [S.PagedCache(k, v, order[None]) for k, v in s["layers"]]
        return s
    ps = case["page"]
    if case["op"] == "update":
        lens = _beam_lengths(case)[0]
        prefix, width, n_pages = _update_pages(case)
        s["layers"] = _layers(case, gen, n_pages)
        table, at = [], case["groups"] * prefix
        for i, n in enumerate(lens):
            mine = -(-n // ps) - prefix
            first = i // case["beams"] * prefix
            table.append(list(range(first, first + prefix)) + list(range(at, at + mine)) + [-1] * (width - prefix - mine))
            at += mine
        _pool(s, case, width, n_pages, len(lens))
        _fill(s, table, lens, torch.randperm(n_pages, generator=gen, device="cuda"))
        parents = _parents(case)
        s["parents"] = _ints(parents)
        s["keep"] = _ints([0 if p < 0 else lens[p] - case["cut"] for p in parents])
        s["n_new"] = _ints([0 if p < 0 else case["n_new"] for p in parents])
        return s
    lens = _spread(case["len_lo"], case["len_hi"], case["rows"])
    used = [-(-n // ps) for n in lens]
    n_pages, width = sum(used), max(used)
    s["layers"] = _layers(case, gen, n_pages)
    _pool(s, case, width, n_pages, case["rows"])
    even = [i % 2 == 0 for i in range(case["rows"])]
    low, table, at = sum(used[::2]), [], [0, sum(used[::2])]
    for n, e in zip(used, even):                                # the even rows came first, and lie lowest
        table.append(list(range(at[not e], at[not e] + n)) + [-1] * (width - n))
        at[not e] += n
    _fill(s, table, lens, torch.cat([torch.randperm(low, generator=gen, device="cuda"),
                                     low + torch.randperm(n_pages - low, generator=gen, device="cuda")]))
    s["leave"] = [_ints([-1 if e else i for i, e in enumerate(even)]), _ints([i if e else -1 for i, e in enumerate(even)])]
    s["join"] = [_ints([n if e else 0 for n, e in zip(lens, even)]), _ints([0 if e else n for n, e in zip(lens, even)])]
    s["turn"] = 0
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _plain_select(s):
    case, x = s["case"], s["logits"]
    g, b, v, n = case["groups"], case["beams"], case["vocab"], case["n"]
    x = x.double()                                             # 64 bits: ranks next to each other decide what is chosen
    top = x.amax(-1, keepdim=True)
    lse = (x - top).exp_().sum(-1, keepdim=True).log() + top
    score = s["scores"].double()[..., None] + x.sub_(lse)
    done = s["finished"]
    if done is not None:                                       # an ended beam offers itself, once
        score = torch.where(done[..., None], -math.inf, score)
        score[..., 0] = torch.where(done, s["scores"].double(), score[..., 0])
    rank = score
    if s["lengths"] is not None:
        long = s["lengths"] + 1 if done is None else s["lengths"] + (~done).int()
        rank = score / long.double().pow(case["penalty"])[..., None]
    rank = rank.reshape(g, b * v)
    if rank.data_ptr() == score.data_ptr():
        rank = rank.clone()
    score = score.reshape(g, b * v)
    place = torch.arange(b * v, device="cuda")
    outs, base = [], (torch.arange(g, device="cuda") * b)
    for _ in range(n):
        best = rank.amax(-1, keepdim=True)
        at = torch.where(rank == best, place, b * v).amin(-1, keepdim=True)
        some = best > -math.inf
        outs.append((torch.where(some, score.gather(1, at), -math.inf), torch.where(some, at, -1)))
        rank.scatter_(1, at, -math.inf)
    at = torch.cat([o[1] for o in outs], 1)
    some, beam = at >= 0, at.clamp(min=0) // v
    token = at.clamp(min=0) % v
    end = _end(case)
    ended = torch.zeros_like(some)
    if done is not None:
        was = done.gather(1, beam)
        token = torch.where(was, end, token)
        ended = some & (was | (token == end))
    out = {"scores": torch.cat([o[0] for o in outs], 1).float(), "parents": torch.where(some, beam + base[:, None], -1).int(),
           "tokens": torch.where(some, token, -1).int()}
    if done is not None:
        out["finished"] = ended
    if s["lengths"] is not None:
        out["lengths"] = torch.where(some, long.gather(1, beam), 0).int()
    return out


def _end(case):
    """The token that ends a sequence."""
    return case["vocab"] // 2 if case["finished"] else -1


def _plain_reorder(s):
    skip, parents = s["case"]["skip"], s["parents"].long()
    for x in s["state"]:
        x[:, skip:] = x[:, skip:][parents]
    s["history"].copy_(s["history"][parents])
    return s["state"] + [s["history"]]


def _copy_rows(layers, src, dst, rows=None):
    """Pages src -> dst of every layer; with rows only the first so many of each."""
    for kv in layers:
        for x in kv:
            raw = x.view(torch.int16 if x.element_size() == 2 else torch.uint8)
            new = raw[src]
            if rows is not None:
                first = torch.arange(x.shape[2], device="cuda")[None, None, :, None] < rows[:, None, None, None]
                new = torch.where(first, new, raw[dst])
            raw[dst] = new


def _count(refs, pages, use, by):
    """refs[page] += by at the places in use."""
    n = len(refs)
    refs.add_(torch.zeros(n + 1, dtype=torch.int32, device="cuda").index_add_(
        0, torch.where(use, pages, n).reshape(-1), torch.full((pages.numel(),), by, dtype=torch.int32, device="cuda"))[:n])


def _plain_update(s, ps, parents, keep, n_new, layers):
    table, lens, refs = s["table"], s["lens"], s["refs"]
    old, had = table.long(), lens.long()
    b, width = table.shape
    n_pages = len(refs)
    cols = torch.arange(width, device="cuda")[None]
    going = parents >= 0
    src = parents.clamp(min=0).long()
    kept = torch.where(going, had[src] if keep is None else torch.minimum(had[src], keep.long()), 0)
    pages = (kept + ps - 1) // ps
    new = torch.where(cols < pages[:, None], old[src], -1)
    _count(refs, old, cols < ((had + ps - 1) // ps)[:, None], -1)
    _count(refs, new, cols < pages[:, None], 1)
    total = kept + n_new
    after = (total + ps - 1) // ps
    at = (kept // ps).clamp(max=width - 1)
    tail = torch.where((n_new > 0) & (kept % ps != 0), new.gather(1, at[:, None])[:, 0], -1)
    grows = tail >= 0
    same = (tail[:, None] == tail[None]) & grows[:, None]
    earlier = torch.tril(same, diagonal=-1).sum(1)                 # rows before this one that write to the same page
    copied = grows & (earlier < refs[tail.clamp(min=0)].long() - 1)
    first = torch.where(copied, at, pages)
    wants = torch.where(n_new > 0, after - first, 0)
    begin = wants.cumsum(0) - wants
    free = refs == 0
    spot = torch.where(free, free.cumsum(0) - 1, n_pages)
    lowest = torch.full((n_pages + 1,), -1, dtype=torch.int64, device="cuda").scatter_(0, spot, torch.arange(n_pages, device="cuda"))
    fresh = (cols >= first[:, None]) & (cols < (first + wants)[:, None])
    given = lowest[(begin[:, None] + cols - first[:, None]).clamp(0, n_pages)]
    new = torch.where(fresh, given, new)
    _count(refs, new, fresh & (new >= 0), 1)
    _count(refs, tail, copied, -1)
    table.copy_(new)
    lens.copy_(total)
    if layers:
        i = copied.nonzero()[:, 0]
        _copy_rows(layers, tail[i], new[i, at[i]], (kept % ps)[i])


def _plain_compact(s):
    refs, table = s["refs"], s["table"]
    n_pages = len(refs)
    live = refs > 0
    border = int(live.sum())
    page = torch.arange(n_pages, device="cuda")
    dst = page[~live & (page < border)]
    src = page[live & (page >= border)].flip(0)
    _copy_rows(s["layers"], src, dst)
    to = page.clone()
    to[src] = dst
    refs[dst], refs[src] = refs[src], torch.zeros_like(src, dtype=torch.int32)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))


def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2410_21465_amd import shadowkv as S
    if case["op"] == "select":
        if own:
            return S.beam_select(s["logits"], s["scores"], n_out=case["n"], finished=s["finished"], lengths=s["lengths"],
                                 length_penalty=case["penalty"], end_token=_end(case))
        return _plain_select(s)
    if case["op"] == "reorder":
        if own:
            S.reorder_rows([x[:, case["skip"]:] for x in s["state"]] + [s["history"]], s["parents"])
            return s["state"] + [s["history"]]
        return _plain_reorder(s)
    if case["op"] == "copy":
        if own:
            S.pages_copy(s["caches"], s["src"], s["dst"])
        else:
            _copy_rows(s["layers"], s["src"].long(), s["dst"].long())
        return s["layers"]
    if case["op"] == "update":
        if own:
            s["pool"].update(parents=s["parents"], keep_lens=s["keep"], n_new=s["n_new"], caches=s["caches"])
        else:
            _plain_update(s, case["page"], s["parents"], s["keep"], s["n_new"], s["layers"])
    else:
        leave, join = s["leave"][s["turn"]], s["join"][s["turn"]]
        s["turn"] ^= 1                                          # those who joined first leave first
        if own:
            s["pool"].update(parents=leave)
            s["pool"].compact(caches=s["caches"])
            s["pool"].update(n_new=join)
        else:
            stay = torch.arange(case["rows"], device="cuda", dtype=torch.int32)
            _plain_update(s, case["page"], leave, None, torch.zeros_like(join), None)
            _plain_compact(s)
            _plain_update(s, case["page"], stay, None, join, None)
    return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "layers": s["layers"]}


def work(case):
    eb = {"bf16": 2, "fp16": 2, "fp32": 4, "fp8": 1}[case.get("dtype", "bf16")]
    if case["op"] == "select":
        rows, out = case["groups"] * case["beams"], case["groups"] * case["n"]
        return {"bytes": rows * (case["vocab"] * eb + 4) + out * 12, "flops": 4 * rows * case["vocab"]}
    if case["op"] == "reorder":
        parents = _parents(case)
        to = [i for i, p in enumerate(parents) if p >= 0 and p != i]
        row = 2 * case["layers"] * (case["inner"] - case["skip"]) * 2 + 4 * case["tokens"]
        return {"bytes": row * (len(to) + len({parents[i] for i in to})) + 4 * len(parents), "flops": len(to)}
    token = 2 * case["layers"] * case["hkv"] * case["d"] * eb      # of keys and values in all layers
    if case["op"] == "copy":
        return {"bytes": 2 * case["pairs"] * case["page"] * token + 8 * case["pairs"], "flops": case["pairs"]}
    if case["op"] == "update":
        ps, (lens, parents, kept, after) = case["page"], _beam_lengths(case)
        n_pages = _update_pages(case)[2]
        moved = [i for i, p in enumerate(parents) if p != i]
        entries = sum(-(-lens[i] // ps) for i in moved) + sum(-(-kept[i] // ps) for i in moved)
        copied = 0                                                  # tokens in last pages that another row holds as well
        for i, p in enumerate(parents):
            if p >= 0 and p in parents[i + 1:]:
                copied += kept[i] % ps
        return {"bytes": 2 * copied * token + 4 * (entries + n_pages) + 16 * len(parents), "flops": len(parents)}
    ps, lens = case["page"], _spread(case["len_lo"], case["len_hi"], case["rows"])
    used = [-(-n // ps) for n in lens]
    stay, n = sum(used[1::2]), sum(used)
    moves = min(stay, n - stay)                                     # live pages above the border
    return {"bytes": 2 * moves * ps * token + 8 * n, "flops": moves}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] != "select":
        return None
    s = prepare(case, seed)
    g, b, v, n = case["groups"], case["beams"], case["vocab"], case["n"]
    out = {"scores": torch.full((g, n), -math.inf, dtype=torch.float64), "parents": torch.full((g, n), -1, dtype=torch.int32),
           "tokens": torch.full((g, n), -1, dtype=torch.int32)}
    if case["finished"]:
        out["finished"] = torch.zeros(g, n, dtype=torch.bool)
    if case["penalty"]:
        out["lengths"] = torch.zeros(g, n, dtype=torch.int32)
    for i in range(g):
        cand = []                                                  # (-rank, beam, token, score, ended, length)
        for j in range(b):
            base = float(s["scores"][i, j])
            ended = bool(s["finished"][i, j]) if case["finished"] else False
            length = int(s["lengths"][i, j]) if case["penalty"] else 0
            if base == -math.inf:
                continue
            if ended:
                cand.append((-base / (length ** case["penalty"] if case["penalty"] else 1.0), j, _end(case), base, True, length))
                continue
            logp = torch.log_softmax(s["logits"][i, j].double(), 0)
            value, token = torch.sort(logp, descending=True, stable=True)
            for x, t in zip(value[:n].tolist(), token[:n].tolist()):
                score = base + x
                cand.append((-score / ((length + 1) ** case["penalty"] if case["penalty"] else 1.0), j, t, score,
                             t == _end(case), length + 1))
        cand.sort(key=lambda c: c[:3])
        for k, (_, j, t, score, ended, length) in enumerate(cand[:n]):
            out["scores"][i, k], out["parents"][i, k], out["tokens"][i, k] = score, i * b + j, t
            if case["finished"]:
                out["finished"][i, k] = ended
            if case["penalty"]:
                out["lengths"][i, k] = length
    return {k: x.cuda() for k, x in out.items()}
