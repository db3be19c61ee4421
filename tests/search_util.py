"""Plain forms of a search's operators: the choice in 64 bits, and a pool of pages that handles one row after the other."""
import math

import torch

LOGIT_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def choose(logits, scores, n, finished=None, lengths=None, penalty=0.0, scale=1.0, end_token=-1):
    """Per group the best first, from the definition on the CPU: (rank, divisor, parent, token, score, finished, length) of the n best
    of every row, the first n of which are the choice."""
    groups, beams, vocab = logits.shape
    x_all, out = logits.detach().cpu().double(), []
    for g in range(groups):
        cand = []
        for b in range(beams):
            s = float(scores[g, b])
            done = finished is not None and bool(finished[g, b])
            length = int(lengths[g, b]) if lengths is not None else 0
            if not math.isfinite(s):
                continue
            divisor = max(float(length + (not done)), 1.0) ** penalty if penalty else 1.0
            if done:
                cand.append((-s / divisor, b, 0, divisor, end_token, s, True, length))
                continue
            x = x_all[g, b]
            if bool(torch.isnan(x).any()) or bool((x == math.inf).any()) or bool((x == -math.inf).all()):
                continue
            top = x.max()
            rel = (x - top) * scale
            score = s + (rel - torch.log(torch.exp(rel).sum()))
            order = torch.sort(x, descending=True, stable=True).indices[:n]
            for place, t in enumerate(order.tolist()):
                if x[t] > -math.inf:
                    cand.append((-float(score[t]) / divisor, b, place, divisor, t, float(score[t]), t == end_token, length + 1))
        cand.sort(key=lambda c: c[:3])
        out.append([(-c[0], c[3], g * beams + c[1], *c[4:7], c[7] if lengths is not None else 0) for c in cand])
    return out


def check_choice(got, want, slack=0.0):
    """A score is rounded once (half a step of fp32, 2^-24 of it); its sum of exponentials is right to 2^-39, and a few operations in 64 bits on
    numbers of up to 2^10 are off by as much: 2^-38 in all, and slack, for larger logits, 2^-50 of them.  So two ranks of different rows that are
    nearer than 2^-37 (and twice the slack, over the lengths) are not told apart: there, and only there, the other order is right too.
    Everything else is as it is in the definition."""
    n = got["scores"].shape[1]
    cols = {k: v.tolist() for k, v in got.items()}
    for g, cand in enumerate(want):
        of = {(c[2], c[3]): c for c in cand}
        seen = set()
        for i in range(n):
            key = (cols["parents"][g][i], cols["tokens"][g][i])
            score, ended, length = (cols[k][g][i] if k in cols else None for k in ("scores", "finished", "lengths"))
            if i >= len(cand):
                assert key == (-1, -1) and score == -math.inf and not ended and not length, f"group {g}, place {i}: {key} {score}"
                continue
            w = cand[i]
            assert key in of and key not in seen, f"group {g}, place {i}: {key}, not {w[2:4]}"
            seen.add(key)
            c = of[key]
            if key != w[2:4]:
                near = (2.0 ** -37 + 2 * slack) / min(c[1], w[1])
                assert c[2] != w[2] and abs(c[0] - w[0]) <= near, f"group {g}, place {i}: {key} of rank {c[0]}, not {w[2:4]} of {w[0]}"
            if abs(c[4]) > 3.4028235677973366e38:
                assert score == -math.inf
            else:
                assert abs(score - c[4]) <= 2.0 ** -24 * abs(c[4]) + 2.0 ** -38 + slack, f"group {g}, place {i}: {score}, not {c[4]}"
            assert ended is None or bool(ended) == c[5], f"group {g}, place {i}: finished {ended}"
            assert length is None or length == c[6], f"group {g}, place {i}: length {length}, not {c[6]}"


class PlainPool:
    """Lists of pages, lengths and counts, one row after the other."""

    def __init__(self, batch, width, n_pages, ps):
        self.rows, self.lens, self.refs = [[] for _ in range(batch)], [0] * batch, [0] * n_pages
        self.batch, self.width, self.ps, self.n_pages = batch, width, ps, n_pages

    def pages(self, n):
        return -(-n // self.ps)

    def update(self, parents=None, keep=None, n_new=0):
        """Returns the copies (src, dst, tokens) and what each row kept."""
        old, old_lens = [list(r) for r in self.rows], list(self.lens)
        kept = []
        for i in range(self.batch):
            p = i if parents is None else parents[i]
            n = old_lens[p] if 0 <= p < self.batch else 0
            if keep is not None:
                n = min(n, max(keep[i], 0))
            kept.append(n)
            self.rows[i] = old[p][:self.pages(n)] if n else []
        for r in old:
            for page in r:
                if 0 <= page < self.n_pages:
                    self.refs[page] -= 1
        for r in self.rows:
            for page in r:
                if 0 <= page < self.n_pages:
                    self.refs[page] += 1
        before = list(self.refs)
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        moves, stopped = [], False
        for i in range(self.batch):
            g = max(n_new if isinstance(n_new, int) else n_new[i], 0)
            self.lens[i] = kept[i]
            if g == 0 or kept[i] + g > self.width * self.ps:
                continue
            tail = self.rows[i][kept[i] // self.ps] if kept[i] % self.ps else -1
            real = 0 <= tail < self.n_pages
            copy = real and self.refs[tail] > 1
            want = self.pages(kept[i] + g) - self.pages(kept[i]) + copy
            if stopped and (want or (real and before[tail] > 1)):
                continue
            if want > len(free):
                stopped = True
                continue
            if copy:
                page = free.pop(0)
                moves.append((tail, page, kept[i] % self.ps))
                self.refs[tail] -= 1
                self.refs[page] = 1
                self.rows[i][-1] = page
                want -= 1
            for _ in range(want):
                page = free.pop(0)
                self.refs[page] = 1
                self.rows[i].append(page)
            self.lens[i] = kept[i] + g
        return moves, kept

    def compact(self, most):
        used = [p for p in range(self.n_pages) if self.refs[p]]
        holes = [p for p in range(self.n_pages) if not self.refs[p]]
        moves = []
        while holes and used and holes[0] < used[-1] and len(moves) < most:
            moves.append((used.pop(), holes.pop(0)))
        to = dict(moves)
        for src, dst in moves:
            self.refs[dst], self.refs[src] = self.refs[src], 0
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        return moves, max([p + 1 for p in range(self.n_pages) if self.refs[p]], default=0)

    def table(self):
        return torch.tensor([r + [-1] * (self.width - len(r)) for r in self.rows], dtype=torch.int32)


def check_pool(pool, plain):
    assert pool.kv_lens.tolist() == plain.lens
    assert pool.page_refs.tolist() == plain.refs
    assert torch.equal(pool.page_table.cpu(), plain.table())


def put_pool(pool, plain):
    """Sets a pool on the device to what the plain one holds."""
    pool.page_table.copy_(plain.table())
    pool.kv_lens.copy_(torch.tensor(plain.lens, dtype=torch.int32))
    pool.page_refs.copy_(torch.tensor(plain.refs, dtype=torch.int32))


def moves_of(pool):
    n = int(pool.move_count)
    return list(zip(pool.move_src[:n].tolist(), pool.move_dst[:n].tolist(), pool.move_rows[:n].tolist()))
