"""Attention of one new token per sequence over a paged cache in 4 bits against the formulas in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_reference import assert_within, attention, visible
from rows_reference import Rows

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV


def _q(seed, n, width):
    return torch.randn(n, width, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _attend(rows, q, heads, layer=0, seqs=None, window=0, sinks=0, max_tokens=0, scale=0.0, cache=None):
    n, d, h = q.shape[0], rows.d, rows.h
    group, w = heads // h, heads * d
    cache = rows.on(S, DEV) if cache is None else cache
    dq = torch.full((n, w + 8), math.nan, dtype=torch.bfloat16, device=DEV)
    dq[:, :w] = q.to(DEV)
    o, lse = torch.full((n, w + 16), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((n, heads), 7.0, device=DEV)
    listed = None if seqs is None else torch.tensor(seqs, dtype=torch.int32, device=DEV)
    a = S.attn_decode_args(dq, o, n, heads, window, sinks, layer=layer, max_tokens=max_tokens, scale=scale, seqs=listed, lse=lse)
    size = S.sif_attn_decode_workspace_bytes(cache, a)
    work = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    S.set_workspace(a, work, size)
    S.sif_k_attn_decode(cache, a)
    torch.cuda.synchronize()
    assert bool((o[:, w:] == 7.0).all())
    held = {}
    for i in range(n):
        s = i if seqs is None else seqs[i]
        if not 0 <= s < len(rows.lens) or rows.lens[s] == 0:
            assert bool((o[i, :w] == 0).all()) and bool((lse[i] == -math.inf).all())
            continue
        m = rows.lens[s]
        if s not in held:
            got = {x: [rows.get(x, layer, s, t) for t in range(m)] for x in "kv"}
            there = torch.tensor([y is not None for y in got["k"]])
            none = torch.zeros(h, d, dtype=torch.float64)
            held[s] = [torch.stack([none if y is None else y for y in got[x]]) for x in "kv"] + [there]
        k, v, there = held[s]
        seen = visible(1, m, window, sinks)[0] & there
        # (what stands in tokens that are not visible has no influence, NaN neither)
        k, v = k.masked_fill(~seen[:, None, None], 0.0), v.masked_fill(~seen[:, None, None], 0.0)
        for g in range(h):
            c = slice(g * group * d, (g + 1) * group * d)
            val, tol = attention(q[i, c].double().view(group, d), k[:, g], v[:, g], seen[None, :].expand(group, -1), scale if scale else 1 / math.sqrt(d))
            assert_within(o[i, c].view(group, d), val["o"], tol["o"], (i, g, "o"))
            assert_within(lse[i, g * group:(g + 1) * group], val["lse"], tol["lse"], (i, g, "lse"))
    return o, lse


@pytest.mark.parametrize("d,kv,heads,page", [(64, 2, 2, 16), (64, 1, 12, 32), (128, 2, 8, 16), (128, 1, 17, 64), (128, 3, 96, 128), (64, 2, 6, 256)])
def test_lengths_from_none_on(d, kv, heads, page):
    rows = Rows("e2m1", [0, 1, 2, 15, 16, 17, 63, 64, 65, 77, 128, 300], page, kv, d, seed=d + page)
    _attend(rows, _q(1, 12, heads * d), heads, layer=1)
    _attend(rows, _q(2, 5, heads * d), heads, seqs=[11, 3, 99, -1, 11], scale=0.3)


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (40, 3), (100, 70), (64, 500), (5000, 4)])
@pytest.mark.parametrize("page", [16, 64])
def test_windows_and_sinks(window, sinks, page):
    rows = Rows("e2m1", [1, 30, 200, 517, 1000], page, 2, 128, layers=1, seed=window)
    _attend(rows, _q(3, 5, 4 * 128), 4, window=window, sinks=sinks)


@pytest.mark.parametrize("page", [16, 64, 128])
def test_long_sequences_in_several_splits(page):
    rows = Rows("e2m1", [9001, 3, 700, 0], page, 1, 128, layers=1, seed=5)
    cache = rows.on(S, DEV)
    for most in (0, 100, 9001, 100000):                    # (only the division of the work depends on it)
        _attend(rows, _q(4, 4, 8 * 128), 8, max_tokens=most, cache=cache)


@pytest.mark.parametrize("n", [65, 130, 256, 257])
def test_more_blocks_than_run_at_once(n):
    """Where the longest sequences come first: all lengths, many of them alike, none, unknown numbers, listed again."""
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 60, (40,), generator=g).tolist() + [0, 1, 64, 64, 64, 65, 300, 300, 128, 1000]
    rows = Rows("e2m1", lens, 16, 8, 64, layers=1, seed=n)
    seqs = torch.randint(0, len(lens), (n,), generator=g).tolist()
    seqs[3], seqs[n - 1], seqs[n // 2] = -1, len(lens), len(lens) - 1
    _attend(rows, _q(n, n, 8 * 64), 8, seqs=seqs)
    _attend(rows, _q(n, n, 8 * 64), 8, seqs=seqs, window=50, sinks=3)
    everyone = Rows("e2m1", [7] * n, 16, 8, 64, layers=1, seed=1)
    _attend(everyone, _q(n + 1, n, 16 * 64), 16)


def test_pages_that_are_none():
    rows = Rows("e2m1", [100, 64, 40], 16, 2, 64, layers=1, seed=6)
    rows.table[0][2], rows.table[0][6], rows.table[1] = -1, 10 ** 6, [-1] * rows.ld
    o, lse = _attend(rows, _q(5, 3, 4 * 64), 4)
    assert not o[1, :256].any() and bool((lse[1] == -math.inf).all())


def test_what_is_not_visible_has_no_influence():
    """NaN groups, the largest powers and every bit set in tokens behind the end, out of the window and in pages of nobody."""
    rows = Rows("e2m1", [40, 100], 16, 2, 128, layers=1, seed=7)
    cache = rows.on(S, DEV)
    q = _q(6, 2, 4 * 128)
    want = _attend(rows, q, 4, window=20, sinks=2, cache=cache)
    seen = {s: set(range(2)) | set(range(m - 20, m)) for s, m in enumerate(rows.lens)}
    used = {(rows.place(s, t), t % 16) for s in seen for t in seen[s]}
    for p in range(rows.n_pages):
        for t in range(16):
            if (p, t) not in used:
                for x in "kv":
                    rows.code[x][0, p, :, t], rows.power[x][0, p, :, t] = 15, 255 if (p + t) % 2 else 254
    got = _attend(rows, q, 4, window=20, sinks=2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_nan_that_is_visible():
    rows = Rows("e2m1", [50, 50, 50], 16, 1, 64, layers=1, seed=8)
    for x, s in (("k", 0), ("v", 1)):
        rows.power[x][0, rows.place(s, 20), 0, 4, 1] = 255
    cache = rows.on(S, DEV)
    q, o = _q(7, 3, 64).to(DEV), torch.empty(3, 64, dtype=torch.bfloat16, device=DEV)
    a = S.attn_decode_args(q, o, 3, 1)
    S.set_workspace(a, torch.empty(1 << 20, dtype=torch.uint8, device=DEV), 1 << 20)
    S.sif_k_attn_decode(cache, a)
    o = o.cpu()
    assert o[0].isnan().all() and o[1, 32:].isnan().all() and not o[1, :32].isnan().any() and not o[2].isnan().any()


def test_powers_at_their_ends():
    """Keys' powers down to 2^-127 and values' up to 2^100: scores of zero, results far from one."""
    rows = Rows("e2m1", [70], 16, 1, 64, layers=1, seed=9)
    rows.power["k"][:] = torch.randint(0, 3, rows.power["k"].shape, generator=torch.Generator().manual_seed(1)).to(torch.uint8)
    rows.power["v"][:] = torch.randint(220, 228, rows.power["v"].shape, generator=torch.Generator().manual_seed(2)).to(torch.uint8)
    _attend(rows, _q(8, 1, 64), 1)
    rows.power["v"][:] = torch.randint(20, 28, rows.power["v"].shape, generator=torch.Generator().manual_seed(2)).to(torch.uint8)
    rows.power["k"][:] = 127
    _attend(rows, _q(8, 1, 128), 2)


def test_the_same_bits_every_time():
    rows = Rows("e2m1", [3000, 5000, 70], 64, 2, 128, layers=1, seed=11)
    cache, q = rows.on(S, DEV), _q(9, 3, 8 * 128).to(DEV)
    got = []
    for _ in range(3):
        o, lse = torch.empty(3, 1024, dtype=torch.bfloat16, device=DEV), torch.empty(3, 8, device=DEV)
        a = S.attn_decode_args(q, o, 3, 8, lse=lse)
        size = S.sif_attn_decode_workspace_bytes(cache, a)
        S.set_workspace(a, torch.empty(size, dtype=torch.uint8, device=DEV), size)
        S.sif_k_attn_decode(cache, a)
        got.append((o.clone(), lse.clone()))
    assert all(torch.equal(got[0][0], x) and torch.equal(got[0][1], y) for x, y in got[1:])
