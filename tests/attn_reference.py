"""Attention under a window with sinks in 64 bits, element by element with what a kernel that rounds probabilities (and, backward, their
gradients) to bf16 once may be off by, and a paged cache's operations one sequence after the other."""
import math

import torch

HALF = 2.0 ** -8        # half a step of bf16, relative
SLACK = 2.0 ** -10      # fp32 sums of up to some thousand terms, and exponentials of scores that are off by their own fp32 sums


def visible(sq, sk, window, sinks):
    p = torch.arange(sq)[:, None] + sk - sq
    j = torch.arange(sk)[None, :]
    near = p - j < window if window else torch.ones(sq, sk, dtype=torch.bool)
    return (j <= p) & (near | (j < sinks))


def attention(q, k, v, seen, scale, do=None, exact=False):
    """One head: q [sq][d], k and v [sk][d] in float64.  Returns (values, bounds) with the keys o, lse and, given do, dq, dk, dv; exact: the
    row term of the gradients is not taken from the stored o."""
    s = (q @ k.t() * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[:, None]), 0.0)
    o = p @ v
    spread = p @ v.abs()
    # a score is off by what its d products add up to, the sum of exponentials by one rounding per term
    off = (q.abs() @ k.abs().t()).masked_fill(~seen, 0.0).amax(1) * scale * q.shape[1] if k.shape[0] else torch.zeros(q.shape[0])
    val = {"o": o, "lse": lse}
    tol = {"o": (HALF + SLACK) * spread + HALF * o.abs() + 1e-30, "lse": 2.0 ** -24 * (off + k.shape[0] + 8 * (1 + lse.abs().nan_to_num(posinf=0.0)))}
    if do is not None:
        dp, delta = do @ v.t(), (do * o).sum(1, keepdim=True)
        ds = p * (dp - delta) * scale
        # a row term taken from the stored o is off by what that is off, tol["o"]
        e_delta = 0.0 if exact else (do.abs() * tol["o"]).sum(1, keepdim=True)
        e_ds = HALF * ds.abs() + scale * p * (e_delta + SLACK * (do.abs() @ v.abs().t() + (do * o).abs().sum(1, keepdim=True)))
        val |= {"dq": ds @ k, "dk": ds.t() @ q, "dv": p.t() @ do}
        tol |= {"dq": e_ds @ k.abs() + HALF * val["dq"].abs() + 1e-30, "dk": e_ds.t() @ q.abs() + HALF * val["dk"].abs() + 1e-30,
                "dv": (HALF + SLACK) * (p.t() @ do.abs()) + HALF * val["dv"].abs() + 1e-30}
    return val, tol


def heads_attention(q, k, v, heads, kv_heads, d, seen, scale, do=None, exact=False):
    """All heads of one sequence: rows of heads * d (query side) and kv_heads * d (key side) columns; lse as [heads][sq]."""
    n = heads // kv_heads
    one = {"o": torch.zeros(q.shape[0], heads * d, dtype=torch.float64), "lse": torch.zeros(heads, q.shape[0], dtype=torch.float64)}
    if do is not None:
        one |= {"dq": torch.zeros_like(one["o"]), "dk": torch.zeros(k.shape[0], kv_heads * d, dtype=torch.float64), "dv": torch.zeros(k.shape[0], kv_heads * d, dtype=torch.float64)}
    val, tol = one, {x: y.clone() for x, y in one.items()}
    for h in range(heads):
        cq, ck = slice(h * d, h * d + d), slice(h // n * d, h // n * d + d)
        a, b = attention(q[:, cq], k[:, ck], v[:, ck], seen, scale, None if do is None else do[:, cq], exact)
        for into, of in ((val, a), (tol, b)):
            into["o"][:, cq], into["lse"][h] = of["o"], of["lse"]
            if do is not None:
                into["dq"][:, cq] = of["dq"]
                into["dk"][:, ck] += of["dk"]
                into["dv"][:, ck] += of["dv"]
    return val, tol


def assert_within(got, val, tol, what):
    got, val = got.detach().double().cpu(), val.double()
    gone = torch.isinf(val)
    assert torch.equal(got[gone], val[gone]), what
    off = (got - val).abs()[~gone]
    assert not torch.isnan(off).any(), (what, "NaN")
    bad = off > tol[~gone]
    assert not bad.any(), (what, int(bad.sum()), float((off / tol[~gone]).max()), got[~gone][bad][:4].tolist(), val[~gone][bad][:4].tolist())


class Cache:
    """A paged cache's bookkeeping, written out; `moved` collects page copies (from, to)."""

    def __init__(self, n_pages, n_seqs, table_ld, page):
        self.page, self.table_ld, self.n_seqs = page, table_ld, n_seqs
        self.table, self.lengths, self.refs, self.moved = [[-1] * table_ld for _ in range(n_seqs)], [0] * n_seqs, [0] * n_pages, []

    def pages(self, tokens):
        return -(-tokens // self.page)

    def listed(self, seqs, n):
        """(entry, sequence or None): numbers outside the table and what was listed before are left out."""
        got, before = [], set()
        for i in range(n):
            s = seqs[i] if seqs is not None else i
            ok = 0 <= s < self.n_seqs and s not in before
            before.add(s)
            got.append(s if ok else None)
        return got

    def extend(self, seqs, counts, n):
        stood, free, asked, status = list(self.refs), [p for p, r in enumerate(self.refs) if r <= 0], 0, []
        plan = []
        for i, s in enumerate(self.listed(seqs, n)):
            c = counts[i] if counts is not None else 1
            if s is None or c < 0 or self.lengths[s] + c > self.table_ld * self.page:
                status.append(-1)
                continue
            m, copy = self.lengths[s], None
            need = self.pages(m + c) - self.pages(m)
            if c > 0 and m % self.page:
                last = self.table[s][m // self.page]
                if not 0 <= last < len(self.refs):
                    status.append(-1)
                    continue
                if stood[last] > 1:
                    copy, need = last, need + 1
            asked += need
            if need and asked > len(free):
                status.append(-2)
                continue
            plan.append((s, m, c, copy, free[asked - need:asked]))
            status.append(0)
        for s, m, c, copy, new in plan:
            new = list(new)
            if copy is not None:
                self.moved.append((copy, new[0]))
                self.refs[copy] -= 1
                self.table[s][m // self.page] = new[0]
                self.refs[new.pop(0)] = 1
            for j in range(self.pages(m), self.pages(m + c)):
                self.table[s][j] = new[0]
                self.refs[new.pop(0)] = 1
            self.lengths[s] = m + c
        return status

    def fork(self, src, dst):
        status, stood = [], list(self.lengths)
        for i, (a, b) in enumerate(zip(src, dst)):
            bad = not (0 <= a < self.n_seqs and 0 <= b < self.n_seqs) or b in dst[:i] or a in dst or stood[b] != 0
            status.append(-1 if bad else 0)
            if not bad:
                for j in range(self.pages(self.lengths[a])):
                    p = self.table[a][j]
                    self.table[b][j] = p
                    if 0 <= p < len(self.refs):
                        self.refs[p] += 1
                self.lengths[b] = self.lengths[a]
        return status

    def _release(self, s, first, last):
        for j in range(first, last):
            p = self.table[s][j]
            if 0 <= p < len(self.refs):
                self.refs[p] -= 1
            self.table[s][j] = -1

    def free(self, seqs, n):
        for s in self.listed(seqs, n):
            if s is not None:
                self._release(s, 0, self.pages(self.lengths[s]))
                self.lengths[s] = 0

    def trim(self, seqs, n, window, sinks):
        for s in self.listed(seqs, n):
            if s is not None:
                self._release(s, self.pages(min(sinks, self.lengths[s])), max(0, self.lengths[s] - window) // self.page)

    def compact(self):
        total = sum(r > 0 for r in self.refs)
        to = [p for p in range(total) if self.refs[p] <= 0]
        of = [p for p in range(total, len(self.refs)) if self.refs[p] > 0]
        where = dict(zip(of, to))
        for a, b in where.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.moved.append((a, b))
        self.table = [[where.get(p, p) for p in row] for row in self.table]
