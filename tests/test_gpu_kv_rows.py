"""New tokens into a paged cache of every format with the rotation on the way, and back out of it, byte by byte."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from rows_reference import HALF, Rows, frequencies, turned

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV

FORMATS = ["bf16", "e4m3", "e2m1"]


def _x(seed, rows, width):
    return torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _i32(x):
    return None if x is None else torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _wide(x, pad=8, fill=math.nan):
    w = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=torch.bfloat16, device=DEV)
    w[:, :x.shape[1]] = x.to(DEV)
    return w


def _rows_of(rows, seqs, starts, n, count):
    """(row, sequence, position, whether the sequence was listed before) of the rows that are a sequence's."""
    got, before = [], set()
    for i in range(n):
        s = i if seqs is None else seqs[i]
        a, b = (i, i + 1) if starts is None else (starts[i], starts[i + 1])
        ok, again = 0 <= s < len(rows.lens), s in before
        before.add(s)
        for r in range(max(a, 0), min(b, count)):
            if ok:
                got.append((r, s, rows.lens[s] - (b - r), again))
    return got


def _append(rows, layer, heads, seqs, starts, n, count, rot, inter=False, m=1.0, there=False, seed=1, k=None, v=None):
    """One call, and what it must leave behind."""
    h, d = rows.h, rows.d
    q = _x(seed, count, max(heads, 1) * d)
    k, v = _x(seed + 1, count, h * d) if k is None else k, _x(seed + 2, count, h * d) if v is None else v
    f = frequencies(rot)
    rope = S.rope_plan(rot, layout=S.SIF_ROPE_INTERLEAVED if inter else S.SIF_ROPE_HALF, magnitude=m)
    cache = rows.on(S, DEV)
    wq, wk, wv = _wide(q, fill=7.0), _wide(k), _wide(v, 16)
    out = wq if there else _wide(torch.full_like(q, 7.0), 16, 7.0)
    a = S.kv_append_args(wk, wv, n, rows=count, layer=layer, seqs=_i32(seqs), starts=_i32(starts), q=wq if heads else None, q_out=out if heads else None, heads=heads)
    S.sif_k_kv_append(cache, rope, a)
    torch.cuda.synchronize()
    want_q, off_q = q.double() if there else torch.full_like(q, 7.0).double(), torch.zeros(q.shape, dtype=torch.float64)
    slack = {}
    for r, s, pos, again in _rows_of(rows, seqs, starts, n, count):
        if pos < 0:
            continue
        p = torch.tensor([pos])
        if heads:
            val, off = turned(q[r].double().view(1, heads, d), p, f, inter, m)
            want_q[r], off_q[r] = val.flatten(), HALF * val.flatten().abs() + (1 + HALF) * off.flatten() + 1e-38
            off_q[r].view(heads, d)[:, rot:] = 0
        if not again:
            val, off = turned(k[r].double().view(1, h, d), p, f, inter, m)
            rows.put("k", layer, s, pos, val[0])
            rows.put("v", layer, s, pos, v[r].double().view(h, d))
            if rows.place(s, pos) >= 0:
                slack[(rows.place(s, pos), pos % rows.page)] = (val[0], HALF * val[0].abs() + (1 + HALF) * off[0] + 1e-38)
    assert torch.all((out[:, :q.shape[1]].cpu().double() - want_q).abs() <= off_q)
    assert bool((out[:, q.shape[1]:] == 7.0).all())
    if rows.dtype == "bf16":
        # turned keys are rounded to bf16 from fp32: within half a step and what that is off, no more, and everything else is equal
        got = rows.t["k"].cpu()
        for (page, t), (val, off) in slack.items():
            y = got[layer, page, :, t].double()
            assert torch.all((y == val) | ((y - val).abs() <= off) | (y.isnan() & val.isnan()))      # (infinities are equal, their difference is none)
            rows.code["k"][layer, page, :, t] = got[layer, page, :, t]
    rows.check()


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("d,kv,heads,rot,page", [(64, 2, 6, 64, 16), (64, 3, 3, 32, 32), (128, 1, 4, 128, 64), (128, 2, 2, 48, 16), (64, 1, 0, 16, 256), (128, 5, 40, 112, 128)])
def test_one_token_each(dtype, d, kv, heads, rot, page):
    lens = [1, page, page + 1, 77, 2, 3 * page, 40]
    for inter in (False, True):
        rows = Rows(dtype, lens, page, kv, d, seed=rot)
        _append(rows, 1, heads, None, None, len(lens), len(lens), rot, inter, there=inter)
        _append(rows, 0, heads, [5, 0, 3], None, 3, 3, rot, inter, m=1.3, seed=9)


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("inter", [False, True])
def test_prompts_of_unequal_length(dtype, inter):
    lens = [100, 0, 31, 64, 5, 200]
    rows = Rows(dtype, lens, 16, 3, 64, seed=2)
    starts = [2, 47, 47, 78, 80, 85, 140]                 # rows 0, 1 and 140 .. belong to nobody, one sequence gets nothing, one its whole length
    _append(rows, 1, 6, None, starts, 6, 145, 64, inter)
    rows = Rows(dtype, lens, 64, 2, 128, seed=3)
    _append(rows, 0, 2, [5, 2, 0, 3], [0, 199, 230, 300, 301], 4, 301, 96, inter, there=True)


@pytest.mark.parametrize("dtype", FORMATS)
def test_lists_that_leave_rows_out(dtype):
    """Unknown numbers, sequences that are listed twice, tokens in front of the first one and without a page."""
    rows = Rows(dtype, [20, 40, 9, 70], 16, 2, 64, seed=4, spare=4)
    rows.table[1][1], rows.table[3][2] = -1, 10 ** 6
    _append(rows, 1, 4, [1, 9, 1, -1, 0, 3, 0, 2], [0, 40, 43, 50, 52, 60, 100, 103, 120], 8, 120, 64)


@pytest.mark.parametrize("dtype", FORMATS)
def test_special_values(dtype):
    rows = Rows(dtype, [37, 5], 32, 2, 128, seed=5)
    k, v = _x(6, 6, 256), _x(7, 6, 256)
    k[0, 3], v[0, 200], k[1, 40:72], v[2, 0] = math.nan, math.nan, 0.0, -math.inf
    v[3, :64], k[4, 128:] = -0.0, 0.0
    k[2, 100], v[4, 5] = math.inf, 3.3895313892515355e38
    v[5, 0:32], v[5, 32:64] = 2.0 ** -120, 1.2e-38                 # powers near their least
    _append(rows, 0, 0, None, [0, 5, 6], 2, 6, 16, k=k, v=v)      # (what is not finite lies behind the rotated elements)


def test_values_next_to_a_border():
    """Turned keys whose 4-bit codes hang on the last bits: at position 0 nothing is turned, so elements stand on borders exactly, a bf16 step to either side of them, and scaled by a
    magnitude that is no power of two."""
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    rowsv = []
    for up in (1.0, 1 + 2.0 ** -7, 1 - 2.0 ** -8):
        x = torch.cat([ties * up, -ties * up, ties, torch.tensor([7.0, 6.0, 0, 0, 1, 2, 3, 4])]).repeat(2)
        rowsv.append(x)
    for m in (1.0, 1 / 3, 0.7, 2.0 ** 0.5):
        for i, x in enumerate(rowsv):
            rows = Rows("e2m1", [1], 16, 1, 64, layers=1, seed=i)
            _append(rows, 0, 0, None, None, 1, 1, 64, m=m, k=x[None].to(torch.bfloat16), v=x[None].to(torch.bfloat16) * 1.5)


@pytest.mark.parametrize("page,d,kv", [(16, 64, 3), (64, 128, 2), (256, 64, 1)])
def test_writing_into_4_bits_without_a_rotation(page, d, kv):
    lens = [50, 300, 0, 17]
    rows = Rows("e2m1", lens, page, kv, d, seed=8)
    cache = rows.on(S, DEV)
    starts = [0, 50, 50, 53, 69]
    seqs = [0, 0, 3, 1]                                    # listed twice: the second entry has no rows and changes nothing
    k, v = _x(1, 70, kv * d), _x(2, 70, kv * d)
    S.sif_k_kv_write(cache, 1, _wide(k), _wide(v), _i32(seqs), 4, starts=_i32(starts), rows=70)
    torch.cuda.synchronize()
    for r, s, pos, again in _rows_of(rows, seqs, starts, 4, 70):
        if not again and pos >= 0:
            rows.put("k", 1, s, pos, k[r].double().view(kv, d))
            rows.put("v", 1, s, pos, v[r].double().view(kv, d))
    rows.check()


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("d,kv,page", [(64, 3, 16), (128, 2, 64), (64, 1, 256)])
def test_reading_back(dtype, d, kv, page):
    lens = [45, 0, page, 7, 130]
    rows = Rows(dtype, lens, page, kv, d, seed=9, spare=2)
    if lens[4] > page:
        rows.table[4][0] = -1                              # a page that was given up
    cache = rows.on(S, DEV)
    for layer, seqs, starts, count in ((0, None, [0, 45, 45, 45 + page, 52 + page, 182 + page], 182 + page), (1, [4, 0, 9, 4, 3], [1, 4, 60, 62, 70, 79], 90), (1, None, None, 5)):
        k, v = _wide(torch.full((count, kv * d), 5.0), 8, 5.0), _wide(torch.full((count, kv * d), 5.0), 24, 5.0)
        n = 5
        S.sif_k_kv_read(cache, layer, k, v, _i32(seqs), n, starts=_i32(starts), rows=count)
        torch.cuda.synchronize()
        want = {x: torch.full((count, kv * d), 5.0, dtype=torch.float64) for x in "kv"}
        for r, s, pos, _ in _rows_of(rows, seqs, starts, n, count):
            for x in "kv":
                y = rows.get(x, layer, s, pos)
                want[x][r] = 0.0 if y is None else y.flatten()
        for x, got in (("k", k), ("v", v)):
            y = got[:, :kv * d].cpu().double()
            if dtype == "e4m3":      # a product in fp32, then one rounding
                assert torch.all((y - want[x]).abs() <= (HALF + 2.0 ** -23) * want[x].abs() + 2.0 ** -134)
            else:
                assert torch.equal(y, want[x]), (x, layer)
            assert bool((got[:, kv * d:] == 5.0).all())
        rows.check("untouched")


@pytest.mark.parametrize("dtype", FORMATS)
def test_as_many_heads_as_there_may_be(dtype):
    rows = Rows(dtype, [3, 18], 16, 1024, 64, layers=2, seed=21)
    _append(rows, 1, 1024, None, [0, 2, 3], 2, 3, 64)
    rows = Rows(dtype, [1], 16, 1, 64, seed=22)
    _append(rows, 0, 1024, None, None, 1, 1, 16, True, there=True)


@pytest.mark.parametrize("dtype", FORMATS)
def test_lists_as_long_as_they_may_be(dtype):
    """One call with 16384 entries, of which some are unknown or listed before, leaves what calls with 512 of them and without those leave; so too reading back, where sequences may be listed again."""
    n, page, d, heads, g = 16384, 16, 64, 2, torch.Generator().manual_seed(23)
    lens = torch.randint(2, 33, (n,), generator=g).int()
    table = torch.randperm(2 * n, generator=g).int().view(n, 2)
    table = torch.where(lens[:, None] > torch.tensor([0, page]), table, -1)
    seqs = torch.randperm(n, generator=g).int()
    seqs[16000], seqs[16383], seqs[700], seqs[9000], seqs[12345] = seqs[3], seqs[16382], seqs[699], -1, n
    count = torch.randint(0, 3, (n,), generator=g)
    count[[3, 16000, 16382, 16383, 699, 700, 9000, 12345]] = 2
    starts = torch.cat([torch.zeros(1, dtype=torch.long), count.cumsum(0)]).int() + 5
    rows = int(starts[-1]) + 3
    q, k, v = (_x(24 + i, rows, w).to(DEV) for i, w in enumerate((heads * d, d, d)))
    rope = S.rope_plan(d)
    kind = {"bf16": S.SIF_BF16, "e4m3": S.SIF_E4M3, "e2m1": S.SIF_E2M1}[dtype]

    def pool(*shape):
        of = {"bf16": (shape, torch.bfloat16), "e4m3": (shape, torch.uint8), "e2m1": (shape[:3] + (page * d * 17 // 32,), torch.uint8)}[dtype]
        return torch.zeros(of[0], dtype=of[1], device=DEV)
    held = []
    for _ in range(2):
        kp, vp = pool(1, 2 * n, 1, page, d), pool(1, 2 * n, 1, d, page)
        t = (kp, vp, table.to(DEV), lens.to(DEV), torch.ones(2 * n, dtype=torch.int32, device=DEV))
        held.append((t, S.kv_cache(*t, kind, page), torch.full_like(q, 7.0)))
    listed, at = seqs.to(DEV), starts.to(DEV)
    S.sif_k_kv_append(held[0][1], rope, S.kv_append_args(k, v, n, rows=rows, seqs=listed, starts=at, q=q, q_out=held[0][2], heads=heads))
    first = {}
    again = torch.zeros(n, dtype=torch.bool)
    for i, s in enumerate(seqs.tolist()):
        again[i] = s in first
        first[s] = i
    assert int(again.sum()) == 3
    alone = torch.where(again, -1, seqs).to(DEV)
    for lo in range(0, n, 512):
        a, b = int(starts[lo]), int(starts[lo + 512])
        S.sif_k_kv_append(held[1][1], rope, S.kv_append_args(k[a:], v[a:], 512, rows=b - a, seqs=alone[lo:lo + 512], starts=at[lo:lo + 513] - a, q=q[a:], q_out=held[1][2][a:], heads=heads))
    torch.cuda.synchronize()
    for x, y in zip(held[0][0], held[1][0]):
        assert torch.equal(x, y)
    twice = torch.zeros(rows, dtype=torch.bool)
    for i in again.nonzero().flatten().tolist():
        twice[int(starts[i]):int(starts[i + 1])] = True
    assert int(twice.sum()) == 6 and torch.equal(held[0][2][~twice.to(DEV)], held[1][2][~twice.to(DEV)])
    assert not bool((held[0][2][twice.to(DEV)] == 7.0).any()) and bool((held[0][2][:5] == 7.0).all()) and bool((held[0][2][rows - 3:] == 7.0).all())
    out = [torch.full((rows, d), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    S.sif_k_kv_read(held[0][1], 0, out[0], out[1], listed, n, starts=at, rows=rows)
    for lo in range(0, n, 512):
        a, b = int(starts[lo]), int(starts[lo + 512])
        S.sif_k_kv_read(held[0][1], 0, out[2][a:], out[3][a:], listed[lo:lo + 512], 512, starts=at[lo:lo + 513] - a, rows=b - a)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    # (values come back as they were written: in bf16 the same, of sequences that are listed once)
    if dtype == "bf16":
        known = torch.zeros(rows, dtype=torch.bool)
        for i in range(n):
            if 0 <= int(seqs[i]) < n and not again[i]:
                known[int(starts[i]):int(starts[i + 1])] = True
        assert torch.equal(out[1][known.to(DEV)], v[known.to(DEV)])


@pytest.mark.parametrize("dtype", FORMATS)
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_long_prompts_in_long_pages(dtype, page):
    """More rows than eight pages have, in one call and sequence by sequence: the same bytes, and back as they went in."""
    lens, d, kv, heads = [3001, 1, 0, 1500, 4097], 64, 3, 4
    per = [-(-m // page) for m in lens]
    total, ld, rows = sum(per), max(per), sum(lens)
    order = torch.randperm(total, generator=torch.Generator().manual_seed(page)).int()
    table, at = torch.full((len(lens), ld), -1, dtype=torch.int32), 0
    for i, m in enumerate(per):
        table[i, :m] = order[at:at + m]
        at += m
    starts = torch.tensor([0] + lens).cumsum(0).int()
    q, k, v = (_x(31 + i, rows, w).to(DEV) for i, w in enumerate((heads * d, kv * d, kv * d)))
    rope, kind = S.rope_plan(32), {"bf16": S.SIF_BF16, "e4m3": S.SIF_E4M3, "e2m1": S.SIF_E2M1}[dtype]
    got = []
    for one in (True, False):
        shape = (1, total, kv, page * d * 17 // 32) if dtype == "e2m1" else None
        kp, vp = (torch.zeros(shape or x, dtype=torch.bfloat16 if dtype == "bf16" else torch.uint8, device=DEV) for x in ((1, total, kv, page, d), (1, total, kv, d, page)))
        t = (kp, vp, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.ones(total, dtype=torch.int32, device=DEV))
        cache, out = S.kv_cache(*t, kind, page), torch.zeros_like(q)
        if one:
            S.sif_k_kv_append(cache, rope, S.kv_append_args(k, v, len(lens), rows=rows, starts=starts.to(DEV), q=q, q_out=out, heads=heads))
        else:
            for i, m in enumerate(lens):
                a = int(starts[i])
                if m:
                    S.sif_k_kv_append(cache, rope, S.kv_append_args(k[a:], v[a:], 1, rows=m, seqs=_i32([i]), starts=_i32([0, m]), q=q[a:], q_out=out[a:], heads=heads))
        kr, vr = torch.zeros_like(k), torch.zeros_like(v)
        S.sif_k_kv_read(cache, 0, kr, vr, None, len(lens), starts=starts.to(DEV), rows=rows)
        torch.cuda.synchronize()
        got.append((kp, vp, out, kr, vr))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    kr, vr = got[0][3:]
    if dtype == "bf16":
        assert torch.equal(vr, v)
    step = {"bf16": 0.0, "e4m3": 2.0 ** -4, "e2m1": 0.25}[dtype]
    # half a step, relative: of the value in 8 bits (2^-10 below its least power); in 4 bits, where the largest of 32 is m 2^e, 3.5 < m <= 7, half a step is at most 2^e, and only where m > 4,
    # so a quarter of the largest
    big = v.cpu().double().abs().view(rows, -1, 32).amax(-1, keepdim=True) if dtype == "e2m1" else v.cpu().double().abs().view(rows, -1, 32)
    assert torch.all((vr.cpu().double() - v.cpu().double()).view(rows, -1, 32).abs() <= step * big + 2.0 ** -10)
    pos = torch.cat([torch.arange(m) for m in lens])
    val, off = turned(k.cpu().double().view(rows, kv, d), pos, frequencies(32), False)
    big = val.abs().view(rows, -1, 32).amax(-1, keepdim=True) if dtype == "e2m1" else val.abs().view(rows, -1, 32)
    half = step if dtype != "bf16" else HALF
    assert torch.all((kr.cpu().double().view_as(val) - val).view(rows, -1, 32).abs() <= half * big + off.view(rows, -1, 32) * 2 + 2.0 ** -10)


def test_4_bit_pages_are_copied_whole():
    """Forking, extending, copying and compacting move powers along with what they belong to."""
    rows = Rows("e2m1", [20, 70, 0, 0], 32, 3, 64, layers=2, seed=10, spare=5, wider=2)
    cache = rows.on(S, DEV)
    size = S.sif_kv_workspace_bytes(cache)
    work = torch.empty(size, dtype=torch.uint8, device=DEV)
    S.sif_k_kv_fork(cache, _i32([0, 1]), _i32([2, 3]), 2)
    S.sif_k_kv_extend(cache, _i32([2, 3]), _i32([1, 1]), 2, work, size)
    S.sif_k_kv_free(cache, _i32([0]), 1)
    S.sif_k_kv_compact(cache, work, size)
    for layer in (0, 1):
        for seq, of, m in ((2, 0, 20), (3, 1, 70), (1, 1, 70)):
            k, v = torch.empty(m, 192, dtype=torch.bfloat16, device=DEV), torch.empty(m, 192, dtype=torch.bfloat16, device=DEV)
            extra = 0 if seq == 1 else 1
            k1, v1 = torch.empty(m + extra, 192, dtype=torch.bfloat16, device=DEV), torch.empty(m + extra, 192, dtype=torch.bfloat16, device=DEV)
            S.sif_k_kv_read(cache, layer, k1, v1, _i32([seq]), 1, starts=_i32([0, m + extra]), rows=m + extra)
            k, v = k1[:m].cpu().double(), v1[:m].cpu().double()
            for t in range(m):
                assert torch.equal(k[t], rows.get("k", layer, of, t).flatten()) and torch.equal(v[t], rows.get("v", layer, of, t).flatten()), (seq, t)


def test_a_pool_past_4_gib_in_4_bits():
    """Pages whose bytes begin beyond 32 bits, in keys and values."""
    d, kv, page = 128, 8, 256
    n_pages = (1 << 32) // (kv * page * d * 17 // 32) + 40
    k, v = (torch.zeros(1, n_pages, kv, page * d * 17 // 32, dtype=torch.uint8, device=DEV) for _ in range(2))
    table = torch.tensor([[n_pages - 1, 3]], dtype=torch.int32, device=DEV)
    lengths, refs = torch.tensor([page + 2], dtype=torch.int32, device=DEV), torch.ones(n_pages, dtype=torch.int32, device=DEV)
    cache = S.kv_cache(k, v, table, lengths, refs, S.SIF_E2M1, page)
    x, y = _x(1, page + 2, kv * d), _x(2, page + 2, kv * d)
    S.sif_k_kv_append(cache, S.rope_plan(16), S.kv_append_args(x.to(DEV), y.to(DEV), 1, rows=page + 2, starts=_i32([0, page + 2])))
    a, b = torch.empty(page + 2, kv * d, dtype=torch.bfloat16, device=DEV), torch.empty(page + 2, kv * d, dtype=torch.bfloat16, device=DEV)
    S.sif_k_kv_read(cache, 0, a, b, None, 1, starts=_i32([0, page + 2]), rows=page + 2)
    from rows_reference import from_e2m1, to_e2m1
    assert torch.equal(b.cpu().double(), from_e2m1(*to_e2m1(y.double().view(page + 2, kv, d))).flatten(1))
    val, _ = turned(x.double().view(page + 2, kv, d), torch.arange(page + 2), frequencies(16), False)
    assert torch.equal(a.cpu().double(), from_e2m1(*to_e2m1(val)).flatten(1))
    assert not k[0, :3].any() and not v[0, 4:n_pages - 1].any()
