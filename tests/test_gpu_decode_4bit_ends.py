"""Attention over a cache in 4 bits where numbers end: held values and keys past the largest in bf16, queries whose 32 elements differ in their powers or are not finite, powers
that are NaN; and launches of more blocks than run at once whose sequences are cut into splits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from rows_reference import Rows
from test_gpu_decode_4bit import _attend, _q

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV

MOST = 3.3895313892515355e38          # the largest number in bf16: held as 4 * 2^126, an infinity as 6 * 2^126


def _put(rows, x, s, t, d, **elements):
    """Token t of sequence s becomes zeros and the given elements, in all heads."""
    y = torch.zeros(rows.h, rows.d, dtype=torch.float64)
    for at, value in elements.items():
        y[:, int(at[1:])] = value
    rows.put(x, 0, s, t, y)


@pytest.mark.parametrize("d", [64, 128])
def test_a_query_of_zeros_and_keys_past_the_largest(d):
    """Zero times what is held is zero: every token counts alike but those whose keys the other elements of q see."""
    rows = Rows("e2m1", [40], 16, 1, d, layers=1, seed=5)
    _put(rows, "k", 0, 3, d, e3=math.inf, e40=-MOST)
    _put(rows, "k", 0, 17, d, e19=-math.inf)
    q = _q(5, 1, 3 * d).view(3, d)
    q[0] = 0.0
    q[1, 3], q[1, 19], q[1, 40] = 0.0, 0.0, -0.0
    q[2, :32] = 0.0
    q[2, 40] = 0.0
    _attend(rows, q.reshape(1, -1), 3)


@pytest.mark.parametrize("d", [64, 128])
def test_small_queries_and_keys_past_the_largest(d):
    """Products of about one from keys of 2^125 to 2^129 and queries of 2^-126."""
    g = torch.Generator().manual_seed(d)
    rows = Rows("e2m1", [70, 1, 200], 32, 2, d, layers=1, seed=4)
    rows.power["k"][..., 0] = torch.randint(252, 255, rows.power["k"].shape[:-1], generator=g).to(torch.uint8)
    q = _q(4, 3, 4 * d).view(3, 4, d)
    q[..., :32] = ((1 + torch.rand(3, 4, 32, generator=g)) * torch.randint(0, 2, (3, 4, 32), generator=g).mul(2).sub(1) * 2.0 ** -126).to(torch.bfloat16)
    q[:, 1, :32:3], q[:, 3, 32:] = 0.0, 0.0
    _attend(rows, q.flatten(1), 4)
    _attend(rows, q.flatten(1), 4, scale=0.01)


@pytest.mark.parametrize("up", [[-126, 20, 0, -60], [90, -126, -100, 3], [3, None, -120, -7], [None, -126, None, 120], [-40, 41, 2, None]], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_of_q_of_different_powers(d, up):
    """Each 32 of q times a power of two, those of the keys by as much smaller, so that every block counts alike in the scores (some of q are zeros); keys past the largest number in bf16 among them."""
    up = up[:d // 32]
    g = torch.Generator().manual_seed(d)
    rows = Rows("e2m1", [70, 1, 200], 32, 2, d, layers=1, seed=4)
    q = torch.zeros(3, 6, d, dtype=torch.float64)
    for b, e in enumerate(up):
        if e is not None:
            q[:, :, b * 32:b * 32 + 32] = (1 + torch.rand(3, 6, 32, generator=g)) * torch.randint(0, 2, (3, 6, 32), generator=g).mul(2).sub(1) * 2.0 ** e
        byte = torch.randint(-2, 1, rows.power["k"].shape[:-1], generator=g) + 127 - (0 if e is None else e)
        rows.power["k"][..., b] = byte.clamp(0, 254).to(torch.uint8)
    q[:, 1, 5::7] = 0.0
    q[:, 2, ::3] *= 2.0 ** -10                                         # far below their block's largest
    q[:, 3, 1::2] *= 2.0 ** -14
    q[:, 4, 1::2] *= 2.0 ** -16
    q = q.flatten(1).to(torch.bfloat16)
    assert bool(q.isfinite().all())
    _attend(rows, q, 6)
    _attend(rows, q, 6, scale=0.01)


@pytest.mark.parametrize("heads", [1, 20])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_values_past_the_largest_leave_other_elements_alone(d, page, heads):
    """A byte of V is an element and the one sixteen on; what one of them holds is nothing to the other.  Their tokens' scores are far below the largest, so all results are finite."""
    rows = Rows("e2m1", [70, 9, 300], page, 1, d, layers=1, seed=d)
    q = _q(1, 1, d).repeat(3, heads)
    for s, m in enumerate(rows.lens):
        rows.put("k", 0, s, 5, q[:1, :d].double())                     # the largest score, some sqrt(d)
        for t, element in ((2, dict(e3=math.inf)), (7, dict(e40=-math.inf, e41=1.0)), (m - 1, dict(e20=MOST, e3=-MOST)), (m // 2, dict(e63=-MOST, e47=MOST))):
            _put(rows, "k", s, t, d)
            _put(rows, "v", s, t, d, **element)
    assert int(rows.power["v"].max()) == 253
    o, _ = _attend(rows, q, heads)
    assert not bool(o[:, :heads * d].isnan().any())
    _attend(rows, q, heads, window=100, sinks=8)


@pytest.mark.parametrize("d", [64, 128])
def test_values_past_the_largest_in_several_splits(d):
    rows = Rows("e2m1", [9000, 4500], 64, 1, d, layers=1, seed=3)
    q = _q(2, 1, d).repeat(2, 4)
    for s, m in enumerate(rows.lens):
        for t in range(5, m, 64):                                      # the largest score of every step
            rows.put("k", 0, s, t, q[:1, :d].double())
        for t in (7, 2100, m - 1):
            _put(rows, "k", s, t, d)
            _put(rows, "v", s, t, d, e17=math.inf, e34=-MOST)
    _attend(rows, q, 4)


@pytest.mark.parametrize("d", [64, 128])
def test_powers_that_are_nan(d):
    rows = Rows("e2m1", [50, 50, 50], 16, 1, d, layers=1, seed=8)
    last = d // 32 - 1
    for x, s in (("k", 0), ("v", 1)):
        rows.power[x][0, rows.place(s, 20), 0, 4, last] = 255
    _put(rows, "v", 1, 9, d, e1=MOST)                                  # (on the way that the largest numbers take too)
    rows.put("k", 0, 1, 9, torch.zeros(1, d, dtype=torch.float64))
    cache = rows.on(S, DEV)
    q, o = _q(7, 3, d).to(DEV), torch.empty(3, d, dtype=torch.bfloat16, device=DEV)
    a = S.attn_decode_args(q, o, 3, 1)
    S.set_workspace(a, torch.empty(1 << 20, dtype=torch.uint8, device=DEV), 1 << 20)
    S.sif_k_attn_decode(cache, a)
    o = o.cpu()
    assert o[0].isnan().all() and o[1, last * 32:].isnan().all() and not o[1, :last * 32].isnan().any() and not o[2].isnan().any()


@pytest.mark.parametrize("d", [64, 128])
def test_queries_that_are_not_finite(d):
    """They make NaN of their own head's results and of nothing else."""
    rows = Rows("e2m1", [100, 64, 3], 16, 2, d, layers=1, seed=6)
    cache, q = rows.on(S, DEV), _q(6, 3, 8 * d)
    want, lse = _attend(rows, q, 8, cache=cache)
    bad = {(0, 1): math.nan, (0, 6): math.inf, (1, 0): -math.inf, (2, 7): math.nan}
    x = q.clone().view(3, 8, d)
    for (i, h), value in bad.items():
        x[i, h, 37] = value
    x, o, got = x.view(3, -1).to(DEV), torch.empty(3, 8 * d, dtype=torch.bfloat16, device=DEV), torch.empty(3, 8, device=DEV)
    a = S.attn_decode_args(x, o, 3, 8, lse=got)
    S.set_workspace(a, torch.empty(1 << 20, dtype=torch.uint8, device=DEV), 1 << 20)
    S.sif_k_attn_decode(cache, a)
    o = o.view(3, 8, d)
    for i in range(3):
        for h in range(8):
            if (i, h) in bad:
                assert bool(o[i, h].isnan().all()) and bool(got[i, h].isnan()), (i, h)
            else:
                assert torch.equal(o[i, h], want[i, h * d:h * d + d]) and torch.equal(got[i, h], lse[i, h]), (i, h)


def test_powers_at_their_ends_with_heads_of_128():
    """Keys' powers down to 2^-127 and values' up to 2^100: scores of zero, results far from one; one token of the largest numbers that bf16 holds."""
    rows = Rows("e2m1", [70], 16, 1, 128, layers=1, seed=9)
    some = lambda seed, lo, hi: torch.randint(lo, hi, rows.power["k"].shape, generator=torch.Generator().manual_seed(seed)).to(torch.uint8)      # noqa: E731
    rows.power["k"], rows.power["v"] = some(1, 0, 3), some(2, 220, 228)
    _attend(rows, _q(8, 1, 128), 1)
    rows.power["k"][:], rows.power["v"] = 127, some(2, 20, 28)
    _attend(rows, _q(8, 1, 256), 2)
    one = Rows("e2m1", [1], 16, 1, 128, layers=1, seed=10)
    one.power["v"][:] = 252
    _attend(one, _q(9, 1, 256), 2)


@pytest.mark.parametrize("n,most", [(65, 0), (65, 20000), (130, 0)])
def test_more_blocks_than_run_at_once_with_splits(n, most):
    """Table rows of more than 4096 tokens, so that the plan has two splits or three, most sequences too short for them: their other splits have nothing to do."""
    g = torch.Generator().manual_seed(n)
    lens = [5000, 0, 1, 2600] + torch.randint(0, 100, (30,), generator=g).tolist()
    rows = Rows("e2m1", lens, 16, 8 if n == 65 else 4, 64, layers=1, seed=n)
    seqs = torch.randint(0, len(lens), (n,), generator=g).tolist()
    seqs[0], seqs[1], seqs[n // 2], seqs[n - 1] = 0, -1, 3, len(lens)
    heads = 2 * rows.h
    cache = rows.on(S, DEV)
    a = S.attn_decode_args(torch.empty(n, heads * 64, dtype=torch.bfloat16, device=DEV), torch.empty(n, heads * 64, dtype=torch.bfloat16, device=DEV), n, heads, max_tokens=most)
    splits = S.sif_attn_decode_workspace_bytes(cache, a) // (n * heads * (64 + 4) * 4)
    assert splits >= 2 and n * rows.h * splits > 512
    _attend(rows, _q(n, n, heads * 64), heads, seqs=seqs, max_tokens=most, cache=cache)
