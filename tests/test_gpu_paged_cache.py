"""A paged key-value cache on the device: its page operations against the same ones written out sequence by sequence, attention over it
against the formulas in 64 bits, and both as a generating program uses them."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_reference import HALF, Cache, assert_within, attention, heads_attention, visible

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV

E4M3 = torch.float8_e4m3fn


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


class Pool:
    """A cache on the device and what it ought to hold: pages whose contents are known, and the bookkeeping."""

    def __init__(self, seed, n_pages, n_seqs, table_ld, page, layers=2, kv_heads=2, d=64, e4m3=False, scales=True, fill=None):
        g = torch.Generator().manual_seed(seed)
        self.page, self.layers, self.kv_heads, self.d, self.e4m3 = page, layers, kv_heads, d, e4m3
        k, v = torch.randn(layers, n_pages, kv_heads, page, d, generator=g), torch.randn(layers, n_pages, kv_heads, d, page, generator=g)
        if fill is not None:
            k.fill_(fill)
            v.fill_(fill)
        self.k, self.v = ((x * 50).clamp(-448, 448).to(E4M3) if e4m3 else x.to(torch.bfloat16) for x in (k, v))
        self.ks, self.vs = (((torch.rand(layers, kv_heads, generator=g) + 0.5) / 50).to(DEV) if e4m3 and scales else None for _ in range(2))
        self.dk, self.dv = self.k.to(DEV), self.v.to(DEV)
        self.table, self.lengths, self.refs = (torch.empty(*s, dtype=torch.int32, device=DEV) for s in ((n_seqs, table_ld), (n_seqs,), (n_pages,)))
        self.cache = S.kv_cache(self.dk, self.dv, self.table, self.lengths, self.refs, S.SIF_E4M3 if e4m3 else S.SIF_BF16, page, k_scale=self.ks, v_scale=self.vs)
        self.bytes = S.sif_kv_workspace_bytes(self.cache)
        self.work = torch.full((self.bytes,), 0xA5, dtype=torch.uint8, device=DEV)
        self.ref = Cache(n_pages, n_seqs, table_ld, page)
        S.sif_k_kv_reset(self.cache)

    def load(self, table, lengths, refs):
        """Puts bookkeeping in place from outside."""
        for into, x in ((self.table, table), (self.lengths, lengths), (self.refs, refs)):
            into.copy_(torch.tensor(x, dtype=torch.int32).to(DEV))
        self.ref.table, self.ref.lengths, self.ref.refs = [list(r) for r in table], list(lengths), list(refs)

    def raw(self, x):
        return x.view(torch.uint8) if self.e4m3 else x.view(torch.int16)

    def check(self, what=""):
        torch.cuda.synchronize()
        assert self.table.cpu().tolist() == self.ref.table, what
        assert self.lengths.cpu().tolist() == self.ref.lengths, what
        assert self.refs.cpu().tolist() == self.ref.refs, what
        self.move()
        assert torch.equal(self.raw(self.dk).cpu(), self.raw(self.k)), what
        assert torch.equal(self.raw(self.dv).cpu(), self.raw(self.v)), what

    def move(self):
        """The page copies of the last operation (none goes to a page twice, nor from one after it was copied to)."""
        for a, b in self.ref.moved:
            self.raw(self.k)[:, b] = self.raw(self.k)[:, a].clone()
            self.raw(self.v)[:, b] = self.raw(self.v)[:, a].clone()
        self.ref.moved.clear()

    def held(self, x, scale, layer, head):
        """A value as the cache holds it."""
        if not self.e4m3:
            return x.to(torch.bfloat16)
        s = 1.0 if scale is None else scale[layer, head].cpu()
        y = x.float() / s
        return torch.where(y.isnan(), y, y.clamp(-448, 448)).to(E4M3)

    def extend(self, seqs, counts, n):
        status = torch.full((n,), 77, dtype=torch.int32, device=DEV)
        S.sif_k_kv_extend(self.cache, None if seqs is None else _i32(seqs), None if counts is None else _i32(counts), n, self.work, self.bytes, status=status)
        assert status.cpu().tolist() == self.ref.extend(seqs, counts, n)
        self.move()

    def fork(self, src, dst):
        status = torch.full((len(src),), 77, dtype=torch.int32, device=DEV)
        S.sif_k_kv_fork(self.cache, _i32(src), _i32(dst), len(src), status=status)
        assert status.cpu().tolist() == self.ref.fork(src, dst)

    def free(self, seqs, n):
        S.sif_k_kv_free(self.cache, None if seqs is None else _i32(seqs), n)
        self.ref.free(seqs, n)

    def trim(self, seqs, n, window, sinks):
        S.sif_k_kv_trim(self.cache, None if seqs is None else _i32(seqs), n, window, sinks)
        self.ref.trim(seqs, n, window, sinks)

    def compact(self):
        S.sif_k_kv_compact(self.cache, self.work, self.bytes)
        self.ref.compact()
        self.move()

    def write(self, layer, k, v, seqs, n, starts=None):
        """k and v: bf16 rows on the host."""
        pad = 8
        wide = [torch.full((x.shape[0], x.shape[1] + pad), math.nan, dtype=torch.bfloat16, device=DEV) for x in (k, v)]
        for w, x in zip(wide, (k, v)):
            w[:, :x.shape[1]] = x.to(DEV)
        S.sif_k_kv_write(self.cache, layer, *wide, None if seqs is None else _i32(seqs), n, starts=None if starts is None else _i32(starts), rows=k.shape[0])
        torch.cuda.synchronize()
        for i, s in enumerate(self.ref.listed(seqs, n)):
            a, b = (i, i + 1) if starts is None else (starts[i], starts[i + 1])
            if s is None:
                continue
            for r in range(a, b):
                pos = self.ref.lengths[s] - (b - r)
                p = self.ref.table[s][pos // self.page] if pos >= 0 else -1
                if not 0 <= p < len(self.ref.refs):
                    continue
                for h in range(self.kv_heads):
                    c = slice(h * self.d, h * self.d + self.d)
                    self.k[layer, p, h, pos % self.page] = self.held(k[r, c], self.ks, layer, h)
                    self.v[layer, p, h, :, pos % self.page] = self.held(v[r, c], self.vs, layer, h)

    def tokens(self, layer, s, h):
        """Keys and values of a sequence's tokens in float64, and which of them have a page."""
        n = self.ref.lengths[s]
        k, v, there = torch.zeros(n, self.d, dtype=torch.float64), torch.zeros(n, self.d, dtype=torch.float64), torch.zeros(n, dtype=torch.bool)
        for t in range(n):
            p = self.ref.table[s][t // self.page]
            if 0 <= p < len(self.ref.refs):
                there[t] = True
                k[t], v[t] = self.k[layer, p, h, t % self.page].double(), self.v[layer, p, h, :, t % self.page].double()
        if self.ks is not None:
            k, v = k * self.ks[layer, h].double().cpu(), v * self.vs[layer, h].double().cpu()
        return k, v, there

    def attend(self, q, heads, layer, seqs, window, sinks, max_tokens=0, scale=0.0):
        """Attention of the rows q (host, bf16) against the reference."""
        n = q.shape[0]
        w = heads * self.d
        dq = torch.full((n, w + 8), math.nan, dtype=torch.bfloat16, device=DEV)
        dq[:, :w] = q.to(DEV)
        o, lse = torch.full((n, w + 16), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((n, heads), 7.0, device=DEV)
        listed = None if seqs is None else _i32(seqs)
        a = S.attn_decode_args(dq, o, n, heads, window, sinks, layer=layer, max_tokens=max_tokens, scale=scale, seqs=listed, lse=lse)
        size = S.sif_attn_decode_workspace_bytes(self.cache, a)
        work = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
        S.set_workspace(a, work, size)
        S.sif_k_attn_decode(self.cache, a)
        torch.cuda.synchronize()
        assert bool((o[:, w:] == 7.0).all())
        group = heads // self.kv_heads
        for i in range(n):
            s = i if seqs is None else seqs[i]
            for h in range(self.kv_heads):
                rows = slice(h * group * self.d, (h + 1) * group * self.d)
                if not 0 <= s < self.ref.n_seqs or self.ref.lengths[s] == 0:
                    assert bool((o[i, rows] == 0).all()) and bool((lse[i, h * group:(h + 1) * group] == -math.inf).all())
                    continue
                k, v, there = self.tokens(layer, s, h)
                seen = visible(1, k.shape[0], window, sinks)[0] & there
                val, tol = attention(q[i, rows].double().view(group, self.d), k, v, seen[None, :].expand(group, -1), scale if scale else 1 / math.sqrt(self.d))
                assert_within(o[i, rows].view(group, self.d), val["o"], tol["o"], (i, h, "o"))
                assert_within(lse[i, h * group:(h + 1) * group], val["lse"], tol["lse"], (i, h, "lse"))
        return o, lse


def _rows(seed, n, width):
    return torch.randn(n, width, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _filled(seed, lens, page, spare=3, wider=0, **kw):
    """Sequences of the given lengths on pages in no order."""
    need = [-(-m // page) for m in lens]
    n_pages, table_ld = sum(need) + spare, max(max(need), 1) + wider
    pool = Pool(seed, n_pages, len(lens), table_ld, page, **kw)
    order = list(range(n_pages))
    random.Random(seed).shuffle(order)
    table, refs, at = [], [0] * n_pages, 0
    for m in need:
        table.append(order[at:at + m] + [-1] * (table_ld - m))
        at += m
    for p in order[:at]:
        refs[p] = 1
    pool.load(table, lens, refs)
    return pool


# ---- page operations -----------------------------------------------------------------------------------------------
def test_extend_takes_the_lowest_pages_in_the_order_of_the_list():
    pool = Pool(1, 12, 5, 4, 16)
    pool.check()
    pool.extend([3, 0], [17, 16], 2)
    pool.check()
    assert pool.ref.table[3][:2] == [0, 1] and pool.ref.table[0][0] == 2
    pool.extend([0, 3, 1], [1, 15, 0], 3)          # a page more, the rest of a page, nothing
    pool.check()
    pool.extend(None, None, 5)                     # one token for everybody
    pool.check()


def test_extend_refuses_entry_by_entry():
    pool = Pool(2, 6, 4, 3, 16)
    pool.extend([0, 9, 0, -1, 1, 2, 3], [20, 1, 5, 1, -3, 49, 48], 7)     # unknown, twice, negative, a row too short, and one that just fits
    pool.check()
    pool.extend([1, 2, 0], [40, 1, 12], 3)         # one page is left: 1 does not fit, then 2 does not either, 0 needs none
    pool.check()
    pool.extend([2], [1], 1)
    pool.check()
    table = [list(r) for r in pool.ref.table]
    table[0][1] = 99                               # a last page that is none
    pool.load(table, pool.ref.lengths[:2] + [1] + pool.ref.lengths[3:], pool.ref.refs)
    table[0][1] = -1
    pool.extend([0, 2], [0, 3], 2)
    pool.check()
    pool.load([[0, 99, -1], [-1] * 3, [1, -1, -1], [-1] * 3], [20, 0, 5, 0], [1, 1, 0, 0, 0, 0])
    pool.extend([0, 2], [1, 1], 2)
    pool.check()


def test_a_shared_last_page_is_copied_when_written_to():
    pool = _filled(3, [20, 32, 0, 0, 0], 16, spare=6, wider=2)
    pool.fork([0, 0, 1], [2, 3, 4])
    pool.check()
    pool.extend([2, 4], [1, 1], 2)                 # 2 copies its half-full page, 4 begins one of its own
    pool.check("after the first")
    pool.extend([3, 0], [0, 13], 2)
    pool.check("after the second")
    pool.extend([3], [1], 1)
    pool.check("alone with its page again")


def test_two_that_share_a_page_and_write_to_it_in_the_same_call():
    pool = _filled(4, [5, 0], 16, spare=4)
    pool.fork([0], [1])
    pool.extend([1, 0], [2, 2], 2)                 # both see a shared page: both copy, and the old one is free
    pool.check()
    assert sum(r > 0 for r in pool.ref.refs) == 2


def test_fork_refuses_entry_by_entry():
    pool = _filled(5, [20, 7, 0, 0, 3, 0], 16)
    pool.fork([0, 1, 0, 6, 0, -1, 4], [2, 2, 4, 3, 9, 3, 4])      # fine, dst twice, dst not empty, no src, no dst, no src, itself
    pool.check()
    pool.fork([0, 3, 5], [3, 5, 1])                # sources that are destinations too
    pool.check()


def test_free_and_trim():
    pool = _filled(6, [200, 64, 1, 17, 0], 16)
    pool.fork([0], [4])
    pool.trim([0, 4, 0, 1, 77], 5, window=40, sinks=3)
    pool.check("trimmed")
    pool.trim([0, 1, 2, 3], 4, window=1, sinks=0)
    pool.check("to the last page")
    pool.free([0, 0, 4, -5, 2], 5)
    pool.check("freed")
    pool.free(None, 5)
    pool.check("all freed")
    assert not any(pool.ref.refs)


@pytest.mark.parametrize("e4m3,page,n_pages", [(False, 16, 40), (True, 64, 7), (False, 32, 17000)])
def test_compact(e4m3, page, n_pages):
    rng = random.Random(n_pages)
    n_seqs, table_ld = 6, max(1, n_pages // 8)
    pool = Pool(7, n_pages, n_seqs, table_ld, page, layers=1 if n_pages > 100 else 3, kv_heads=1, d=64, e4m3=e4m3)
    pages = rng.sample(range(n_pages), n_seqs * table_ld // 2)
    refs, table = [0] * n_pages, []
    for s in range(n_seqs):
        mine = [pages.pop() for _ in range(len(pages) // (n_seqs - s))]
        table.append(mine + [-1] * (table_ld - len(mine)))
        for p in mine:
            refs[p] = 1
    table[0] = list(table[1])                      # shared pages
    refs = [0] * n_pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    lengths = [sum(p >= 0 for p in row) * page for row in table]
    if lengths[2] > page:
        refs[table[2][0]] -= 1
        table[2][0] = -1                           # a page given up
    pool.load(table, lengths, refs)
    pool.compact()
    pool.check()
    used = sum(r > 0 for r in pool.ref.refs)
    assert all(r > 0 for r in pool.ref.refs[:used])
    pool.compact()                                 # nothing left to do
    pool.check()


def test_compact_of_an_empty_and_a_full_pool():
    pool = Pool(8, 5, 2, 5, 16)
    pool.compact()
    pool.check("empty")
    pool.extend([0], [80], 1)
    pool.compact()
    pool.check("full")


@pytest.mark.parametrize("e4m3", [False, True])
def test_copy_pages(e4m3):
    pool = Pool(9, 10, 1, 1, 128, kv_heads=3, d=128, e4m3=e4m3)
    src, dst = [0, 1, 0, 3, 10, 5, -1, 6, 8], [4, 5, 7, 4, 2, 2, 2, 6, 9]
    status = torch.full((len(src),), 77, dtype=torch.int32, device=DEV)
    S.sif_k_kv_copy_pages(pool.cache, _i32(src), _i32(dst), len(src), status=status)
    want = []
    for i, (a, b) in enumerate(zip(src, dst)):
        bad = not (0 <= a < 10 and 0 <= b < 10) or b in dst[:i] or a in dst
        want.append(-1 if bad else 0)
        if not bad:
            pool.ref.moved.append((a, b))
    assert status.cpu().tolist() == want and 0 in want
    pool.check()


def test_a_long_list_on_a_large_pool():
    """1024 sequences at once, pages found over more than one turn of the search."""
    rng = random.Random(11)
    pool = Pool(10, 20001, 1024, 40, 16, layers=1, kv_heads=1, d=64)
    for k in range(3):
        seqs = rng.sample(range(1024), 1024)
        pool.extend(seqs, [rng.randint(0, 150) for _ in seqs], 1024)
    pool.check()
    pool.free(rng.sample(range(1024), 500), 500)
    gone = [s for s in range(1024) if pool.ref.lengths[s] == 0][:200]
    kept = [s for s in range(1024) if pool.ref.lengths[s] > 0][:200]
    pool.fork(kept, gone)
    pool.extend(gone, [rng.randint(1, 40) for _ in gone], len(gone))
    pool.check()
    assert pool.ref.lengths[gone[0]] > 0


@pytest.mark.parametrize("e4m3,page", [(False, 16), (True, 32)])
def test_operations_one_after_the_other(e4m3, page):
    rng = random.Random(12 + page)
    pool = Pool(13, 60, 12, 9, page, e4m3=e4m3)
    for turn in range(60):
        pick, n = rng.random(), rng.randint(1, 8)
        seqs = [rng.randint(-1, 12) for _ in range(n)]
        if pick < 0.45:
            pool.extend(seqs, [rng.choice((0, 1, 1, 5, page, rng.randint(0, 3 * page))) for _ in seqs], n)
        elif pick < 0.65:
            pool.fork(seqs, [rng.randint(0, 11) for _ in seqs])
        elif pick < 0.8:
            pool.free(seqs, n)
        elif pick < 0.9:
            pool.trim(seqs, n, rng.randint(1, 3 * page), rng.choice((0, 1, page)))
        else:
            pool.compact()
        pool.check(turn)


@pytest.mark.parametrize("e4m3,page,d,kv_heads,scales", [(False, 16, 64, 3, True), (False, 128, 128, 2, True), (True, 16, 128, 2, True), (True, 256, 64, 1, True), (True, 32, 64, 2, False)])
def test_write(e4m3, page, d, kv_heads, scales):
    lens = [33, 1, 0, 300, 16, 5]
    pool = _filled(14, lens, page, d=d, kv_heads=kv_heads, e4m3=e4m3, scales=scales)
    w = kv_heads * d
    k, v = _rows(1, 6, w), 20 * _rows(2, 6, w)
    pool.write(1, k, v, None, 6)                   # one row each; sequence 2 is empty
    pool.check("one each")
    k[0, 0], k[1, 1], v[3, 2], v[4, 0] = math.nan, 1e30, -math.inf, math.nan
    pool.write(0, k[:5], v[:5], [5, 3, 9, 3, 0], 5)      # unknown, and listed twice
    torch.cuda.synchronize()
    for mine, there in ((pool.k, pool.dk), (pool.v, pool.dv)):
        a, b = mine.float(), there.cpu().float()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    pool.dk.copy_(pool.k.to(DEV))                  # (a NaN has more than one pattern)
    pool.dv.copy_(pool.v.to(DEV))
    starts = [0, 33, 33, 40, 240, 245, 245]        # all of it, nothing, more than there is, a long piece, the last ones
    pool.write(1, _rows(3, 250, w), _rows(4, 250, w), [0, 1, 2, 3, 4, 5], 6, starts=starts)
    pool.check("pieces")
    starts = [3, 20, 21]                           # rows in front of and behind all entries
    pool.write(0, _rows(5, 40, w), _rows(6, 40, w), [3, 1], 2, starts=starts)
    pool.check("some rows")


# ---- attention -----------------------------------------------------------------------------------------------------
DECODE = [
    # lengths, heads, kv heads, d, page, window, sinks, 8 bits
    ([1], 1, 1, 64, 16, 0, 0, False),
    ([0, 1, 2, 31, 32, 33, 0], 4, 4, 64, 16, 0, 0, False),
    ([77], 12, 12, 64, 16, 0, 0, False),
    ([15, 16, 17, 63, 64, 65, 129], 8, 2, 128, 16, 0, 0, False),
    ([15, 16, 17, 63, 64, 65, 129], 8, 2, 128, 32, 0, 0, True),
    ([500, 3, 1000], 6, 2, 64, 64, 100, 4, False),
    ([500, 3, 1000], 6, 2, 64, 256, 100, 4, True),
    ([300, 41, 90], 32, 1, 64, 16, 0, 0, False),           # more query heads than a tile has
    ([300, 41, 90], 40, 2, 128, 16, 33, 0, True),
    ([700, 40, 33], 4, 2, 128, 16, 1, 0, False),           # the newest token alone
    ([700, 40, 33], 4, 2, 128, 16, 1, 1, True),
    ([900, 64, 65, 200], 4, 1, 64, 128, 40, 70, False),    # sinks of more than a step, and up to the window
    ([900, 64, 65, 200], 4, 1, 64, 128, 40, 5000, False),
    ([900, 64, 65, 200], 4, 1, 128, 16, 500, 33, True),
    ([1000, 999], 2, 2, 64, 32, 5000, 4, False),           # a window past the sequence
]


@pytest.mark.parametrize("lens,heads,kv_heads,d,page,window,sinks,e4m3", DECODE)
@pytest.mark.parametrize("hint", [0, 1, 100000])
def test_decode(lens, heads, kv_heads, d, page, window, sinks, e4m3, hint):
    """hint: what the call is told of the lengths - nothing, far too little, far too much; only the division of the work may depend on it."""
    pool = _filled(sum(lens) + heads, lens, page, kv_heads=kv_heads, d=d, e4m3=e4m3)
    pool.attend(_rows(3, len(lens), heads * d), heads, 1, None, window, sinks, max_tokens=hint)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_lists_holes_and_garbage(e4m3):
    """A list with repetitions and numbers outside the table, rows with entries that are no pages, free pages and the rest of last pages
    full of NaN, lengths beyond the row and below zero."""
    lens, d, page = [100, 60, 0, 250, 33], 64, 16
    pool = _filled(20, lens, page, kv_heads=2, d=d, e4m3=e4m3, spare=5)
    for p, r in enumerate(pool.ref.refs):
        if r == 0:
            pool.k[:, p], pool.v[:, p] = math.nan, math.nan
    for s, m in enumerate(lens):
        if m % page:
            p = pool.ref.table[s][m // page]
            pool.k[:, p, :, m % page:], pool.v[:, p, :, :, m % page:] = math.nan, math.nan
    pool.dk.copy_(pool.k.to(DEV))
    pool.dv.copy_(pool.v.to(DEV))
    table = [list(r) for r in pool.ref.table]
    table[0][2], table[3][4], table[3][5], table[1][1] = -1, 1 << 30, -7, len(pool.ref.refs)
    table[4] = [-1] * len(table[4])                # a sequence without any page
    pool.load(table, pool.ref.lengths, pool.ref.refs)
    seqs = [3, 0, 0, 5, 2, -1, 1, 4, 1 << 30]
    for window, sinks in ((0, 0), (40, 3), (70, 20)):
        for hint in (0, 64):
            pool.attend(_rows(21, len(seqs), 4 * d), 4, 0, seqs, window, sinks, max_tokens=hint)
    p = table[3][250 // page]                      # (all of that page is read from here on)
    pool.k[:, p, :, 250 % page:], pool.v[:, p, :, :, 250 % page:] = 0.5, 0.25
    pool.dk.copy_(pool.k.to(DEV))
    pool.dv.copy_(pool.v.to(DEV))
    most = len(table[0]) * page
    pool.lengths[3], pool.lengths[0] = most + 1000, -4
    pool.ref.lengths[3], pool.ref.lengths[0] = most, 0
    pool.attend(_rows(22, len(seqs), 4 * d), 4, 0, seqs, 0, 0)


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 5)])
def test_decode_with_scales_of_zero_and_below(window, sinks):
    """A key is what is held times its scale, whatever that is: a kv head whose keys are all zero (a scale of 0), and negative ones, in
    lengths that end inside a step."""
    lens, d = [77, 300, 9], 64
    pool = _filled(31, lens, 32, kv_heads=3, d=d, e4m3=True)
    pool.ks[1].copy_(torch.tensor([0.0, -0.02, 0.03]))
    pool.vs[1].copy_(torch.tensor([-0.02, 0.01, 0.0]))
    pool.attend(_rows(32, 3, 6 * d), 6, 1, None, window, sinks)


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_of_a_long_sequence_beside_short_ones(e4m3):
    lens = [20011, 1, 300]
    pool = _filled(23, lens, 64, kv_heads=1, d=128, layers=1, e4m3=e4m3)
    for window, sinks in ((0, 0), (9000, 4)):
        pool.attend(_rows(24, 3, 8 * 128), 8, 0, None, window, sinks, scale=0.2)


def test_decode_past_32_bits():
    """A pool of more than 4 GiB per K and V: the pages at its end, of the last layer."""
    layers, n_pages, kv_heads, page, d = 3, 2800, 8, 256, 128          # 4.4 GB each of K and V
    k = torch.zeros(layers, n_pages, kv_heads, page, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(layers, n_pages, kv_heads, d, page, dtype=torch.bfloat16, device=DEV)
    assert k.numel() * 2 > 1 << 32 and layers * n_pages * kv_heads * page * d > 1 << 31
    table, lengths, refs = _i32([n_pages - 1, n_pages - 2]).view(1, 2), _i32([300]), torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    c = S.kv_cache(k, v, table, lengths, refs, S.SIF_BF16, page)
    new_k, new_v, q = _rows(1, 300, kv_heads * d), _rows(2, 300, kv_heads * d), _rows(3, 1, kv_heads * d)
    S.sif_k_kv_write(c, layers - 1, new_k.to(DEV), new_v.to(DEV), None, 1, starts=_i32([0, 300]), rows=300)
    o, lse = torch.empty(1, kv_heads * d, dtype=torch.bfloat16, device=DEV), torch.empty(1, kv_heads, device=DEV)
    qd = q.to(DEV)
    a = S.attn_decode_args(qd, o, 1, kv_heads, layer=layers - 1, lse=lse, max_tokens=64)
    S.sif_k_attn_decode(c, a)
    torch.cuda.synchronize()
    val, tol = heads_attention(q.double(), new_k.double(), new_v.double(), kv_heads, kv_heads, d, visible(1, 300, 0, 0), 1 / math.sqrt(d))
    assert_within(o, val["o"], tol["o"], "o")
    assert_within(lse.t(), val["lse"], tol["lse"], "lse")
    assert int(k[:layers - 1].count_nonzero()) == 0 and int(k[layers - 1, :n_pages - 2].count_nonzero()) == 0


# ---- together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("e4m3,window,sinks", [(False, 0, 0), (False, 40, 4), (True, 40, 4)])
def test_prompt_then_tokens(e4m3, window, sinks):
    """Prompts go through attention over whole sequences, their keys and values into the cache; answers are forked from them and take
    token after token, trimmed to the window and compacted on the way.  Decoding a prompt's last token gives what the prompt's attention gave."""
    heads, kv_heads, d, page, lens = 4, 2, 64, 16, [70, 33]
    pool = Pool(30, 60, 8, 12, page, layers=1, kv_heads=kv_heads, d=d, e4m3=e4m3)
    starts, w, wk = [0, 70, 103], heads * d, kv_heads * d
    q, k, v = _rows(31, 103, w), _rows(32, 103, wk), _rows(33, 103, wk)
    dq, dk, dv = (x.to(DEV) for x in (q, k, v))
    o = torch.empty_like(dq)
    S.sif_k_window_attn_fwd(S.window_attn_args(dq, dk, dv, o, heads, kv_heads, d, 2, 70, 70, window, sinks, starts=_i32(starts), rows=103))
    pool.extend([0, 1], lens, 2)
    pool.write(0, k, v, [0, 1], 2, starts=starts)
    pool.check("prompts")
    last, _ = pool.attend(q[[69, 102]], heads, 0, [0, 1], window, sinks)
    if not e4m3:
        for i, r in enumerate((69, 102)):          # two computations of the same number, each within a bound of the exact one
            val, tol = heads_attention(q[r:r + 1].double(), k[starts[i]:r + 1].double(), v[starts[i]:r + 1].double(), heads, kv_heads, d,
                                       visible(1, lens[i], window, sinks), 1 / math.sqrt(d))
            for got in (o[r:r + 1], last[i:i + 1, :w]):
                assert_within(got, val["o"], tol["o"], r)
    pool.fork([0, 0, 1], [2, 3, 4])
    live = [0, 1, 2, 3, 4]
    for turn in range(30):
        pool.extend(live, None, len(live))
        pool.write(0, _rows(100 + turn, len(live), wk), _rows(200 + turn, len(live), wk), live, len(live))
        pool.attend(_rows(300 + turn, len(live), w), heads, 0, live, window, sinks, max_tokens=110)
        if window and turn % 7 == 3:
            pool.trim(live, len(live), window, sinks)
        if turn == 11:
            pool.free([3], 1)
            live.remove(3)
        if turn in (12, 25):
            pool.compact()
        pool.check(turn)


def test_a_step_captured_and_replayed():
    """Extension, write and attention of a step as one graph, replayed while the cache grows; eager work between the replays."""
    heads, kv_heads, d, page, n = 4, 2, 64, 16, 3
    pool = _filled(40, [30, 5, 47], page, spare=20, wider=5, layers=1, kv_heads=kv_heads, d=d)
    w, wk = heads * d, kv_heads * d
    q, k, v = (torch.zeros(n, x, dtype=torch.bfloat16, device=DEV) for x in (w, wk, wk))
    o, status = torch.zeros(n, w, dtype=torch.bfloat16, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    a = S.attn_decode_args(q, o, n, heads)
    size = S.sif_attn_decode_workspace_bytes(pool.cache, a)
    work = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)
    S.set_workspace(a, work, size)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream()
        S.sif_k_kv_extend(pool.cache, None, None, n, pool.work, pool.bytes, status=status, stream=s)
        S.sif_k_kv_write(pool.cache, 0, k, v, None, n, stream=s)
        S.sif_k_attn_decode(pool.cache, a, stream=s)
    pool.check("capturing runs nothing")
    for turn in range(20):
        rows = [_rows(turn * 3 + i, n, x) for i, x in enumerate((w, wk, wk))]
        for into, x in zip((q, k, v), rows):
            into.copy_(x.to(DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert pool.ref.extend(None, None, n) == status.cpu().tolist() == [0] * n
        for i in range(n):
            pos = pool.ref.lengths[i] - 1
            p = pool.ref.table[i][pos // page]
            pool.k[0, p, :, pos % page], pool.v[0, p, :, :, pos % page] = rows[1][i].view(kv_heads, d), rows[2][i].view(kv_heads, d)
        pool.check(turn)
        eager, _ = pool.attend(rows[0], heads, 0, None, 0, 0)      # held against the reference, and the replay against it
        assert torch.equal(eager[:, :w], o), turn


def test_two_decodes_at_once():
    """Two calls side by side on streams and workspaces of their own, over one cache."""
    pool = _filled(50, [3000, 2000], 16, layers=1, kv_heads=2, d=128)
    alone, calls = [], []
    for i in range(2):
        q, o = _rows(i, 2, 8 * 128).to(DEV), torch.zeros(2, 8 * 128, dtype=torch.bfloat16, device=DEV)
        a = S.attn_decode_args(q, o, 2, 8, window=[0, 700][i], sinks=4)
        size = S.sif_attn_decode_workspace_bytes(pool.cache, a)
        work = torch.empty(size, dtype=torch.uint8, device=DEV)
        S.set_workspace(a, work, size)
        S.sif_k_attn_decode(pool.cache, a)
        torch.cuda.synchronize()
        alone.append(o.clone())
        o.zero_()
        calls.append((a, q, o, work, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for a, _, _, _, s in calls:
            S.sif_k_attn_decode(pool.cache, a, stream=s)
    torch.cuda.synchronize()
    for want, (_, _, o, _, _) in zip(alone, calls):
        assert torch.equal(want, o)
