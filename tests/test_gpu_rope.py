"""Rotary positions on the GPU against their formulas in 64 bits: layouts, parts of heads, strides, far positions, in place, back, in a graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from rows_reference import HALF, frequencies, turned

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV


def _x(seed, rows, width):
    return torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _wide(x, pad=8):
    """On the device with columns behind each row that nobody may touch."""
    w = torch.full((x.shape[0], x.shape[1] + pad), 7.0, dtype=torch.bfloat16, device=DEV)
    w[:, :x.shape[1]] = x.to(DEV)
    return w


def _check(got, x, pos, f, heads, d, inter, m, back, what):
    rows = x.shape[0]
    val, off = turned(x.double().view(rows, heads, d), pos, f, inter, m, back)
    y = got[:, :heads * d].cpu().double().view(rows, heads, d)
    assert torch.all((y - val).abs() <= HALF * val.abs() + (1 + HALF) * off + 1e-38), (what, float(((y - val).abs() - HALF * val.abs() - off).max()))
    r = 2 * len(f)
    assert torch.equal(y[..., r:], x.double().view(rows, heads, d)[..., r:]), what
    assert bool((got[:, heads * d:] == 7.0).all()), what


CASES = [
    # rows, heads, kv heads, d, rot
    (1, 1, 0, 16, 16), (1, 12, 12, 64, 64), (77, 12, 4, 64, 32), (5, 3, 1, 80, 48), (130, 32, 8, 128, 128), (33, 2, 2, 256, 256), (9, 7, 7, 128, 112), (1000, 1, 1, 64, 16),
    (3, 100, 1, 24, 16), (300, 16, 2, 128, 64),
]


@pytest.mark.parametrize("rows,heads,kv,d,rot", CASES)
@pytest.mark.parametrize("inter", [False, True])
def test_rows_of_heads(rows, heads, kv, d, rot, inter):
    f = frequencies(rot, base=500000.0)
    rope = S.rope_plan(rot, layout=S.SIF_ROPE_INTERLEAVED if inter else S.SIF_ROPE_HALF, base=500000.0, magnitude=1.25)
    q, k = _x(1, rows, heads * d), _x(2, rows, max(kv, 1) * d)
    for back in (False, True):
        for given in (None, "listed"):
            seq, first = max(1, rows // 2), 1000
            pos = torch.arange(rows) % seq + first if given is None else torch.randint(0, 300000, (rows,), generator=torch.Generator().manual_seed(3))
            where = dict(seq=seq, first=first) if given is None else dict(positions=pos.to(torch.int32).to(DEV))
            for there in (False, True):
                wq, wk = _wide(q), _wide(k, 16)
                oq, ok = (wq, wk) if there else (_wide(torch.zeros_like(q), 24), _wide(torch.zeros_like(k)))
                S.sif_k_rope(rope, S.rope_args(wq, oq, rows, heads, d, k=wk if kv else None, k_out=ok if kv else None, kv_heads=kv, inverse=back, **where))
                _check(oq, q, pos, f, heads, d, inter, 1.25, back, ("q", back, given, there))
                if kv:
                    _check(ok, k, pos, f, kv, d, inter, 1.25, back, ("k", back, given, there))
                else:
                    assert torch.equal(ok[:, :k.shape[1]].cpu(), k if there else torch.zeros_like(k))


@pytest.mark.parametrize("d,rot", [(40, 16), (256, 16), (128, 48), (64, 64)])
def test_one_in_place_and_one_not(d, rot):
    rows, heads, kv = 37, 3, 2
    f, rope, pos = frequencies(rot), S.rope_plan(rot), torch.arange(rows)
    q, k = _x(4, rows, heads * d), _x(5, rows, kv * d)
    for q_there in (False, True):
        wq, wk = _wide(q), _wide(k, 16)
        oq, ok = (wq, _wide(torch.zeros_like(k))) if q_there else (_wide(torch.zeros_like(q), 24), wk)
        S.sif_k_rope(rope, S.rope_args(wq, oq, rows, heads, d, k=wk, k_out=ok, kv_heads=kv, seq=rows))
        _check(oq, q, pos, f, heads, d, False, 1.0, False, ("q", q_there))
        _check(ok, k, pos, f, kv, d, False, 1.0, False, ("k", q_there))


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="parts", factor=32.0, trained=4096.0)], ids=str)
def test_scaled_frequencies(kw):
    how = {"linear": "SIF_ROPE_LINEAR", "base": "SIF_ROPE_BASE", "parts": "SIF_ROPE_PARTS"}[kw["scaling"]]
    rope = S.rope_plan(64, scaling=getattr(S, how), factor=kw["factor"], trained_tokens=kw.get("trained", 0.0))
    q = _x(4, 200, 128)
    wq = _wide(q)
    S.sif_k_rope(rope, S.rope_args(wq, wq, 200, 2, 64, seq=200, first=30000))
    _check(wq, q, torch.arange(200) + 30000, frequencies(64, **kw), 2, 64, False, 1.0, False, kw)


def test_far_and_negative_positions():
    pos = torch.tensor([0, 1, -1, 2 ** 20, 10 ** 7, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 123456789])
    q, f, rope = _x(5, len(pos), 64), frequencies(64), S.rope_plan(64)
    wq = _wide(q)
    S.sif_k_rope(rope, S.rope_args(wq, wq, len(pos), 1, 64, positions=pos.to(torch.int32).to(DEV)))
    _check(wq, q, pos, f, 1, 64, False, 1.0, False, "listed")
    wq = _wide(q)
    S.sif_k_rope(rope, S.rope_args(wq, wq, len(pos), 1, 64, seq=9, first=2 ** 31 - 5))      # past 31 bits: counted on, not wrapped
    _check(wq, q, torch.arange(9) + 2 ** 31 - 5, f, 1, 64, False, 1.0, False, "first")


def test_special_values_stay_in_their_pairs():
    q = torch.zeros(2, 64, dtype=torch.bfloat16)
    q[0, 5], q[0, 40], q[1, 63] = float("nan"), float("inf"), float("nan")
    rope = S.rope_plan(32)
    out = torch.zeros(2, 64, dtype=torch.bfloat16, device=DEV)
    S.sif_k_rope(rope, S.rope_args(q.to(DEV), out, 2, 1, 64, seq=2, first=3))
    out = out.cpu()
    assert torch.nonzero(out[0].isnan())[:, 0].tolist() == [5, 21] and out[0, 40] == float("inf") and torch.nonzero(out[1].isnan())[:, 0].tolist() == [63]
    q[0] = 0
    out = torch.ones(2, 64, dtype=torch.bfloat16, device=DEV)
    S.sif_k_rope(S.rope_plan(32, magnitude=0.0), S.rope_args(q.to(DEV), out, 1, 1, 64, seq=1))
    assert not out[0].any() and out[1].eq(1).all()


@pytest.mark.parametrize("inter", [False, True])
def test_gradients(inter):
    """Backward is the transposed matrix, element for element: columns from unit vectors forward, rows from unit vectors back; and the forward pass changes along a direction by
    what the gradient says."""
    d, rot, p = 64, 48, 12345
    rope = S.rope_plan(rot, layout=S.SIF_ROPE_INTERLEAVED if inter else S.SIF_ROPE_HALF, magnitude=1.5)
    eye = torch.eye(d, dtype=torch.bfloat16, device=DEV)
    fwd, bwd = torch.empty_like(eye), torch.empty_like(eye)
    S.sif_k_rope(rope, S.rope_args(eye, fwd, d, 1, d, seq=1, first=p))
    S.sif_k_rope(rope, S.rope_args(eye, bwd, d, 1, d, seq=1, first=p, inverse=True))
    assert torch.equal(fwd.t().contiguous(), bwd) and fwd.count_nonzero() == 2 * rot + (d - rot)
    rows, h = 40, 3
    x, e, dy = _x(6, rows, h * d).to(DEV), _x(7, rows, h * d).to(DEV), _x(8, rows, h * d).to(DEV)
    step = 8.0
    plus, minus = ((x.float() + s * step * e.float()).to(torch.bfloat16) for s in (1, -1))
    out = [torch.empty_like(x) for _ in range(3)]
    for a, b in ((plus, out[0]), (minus, out[1])):
        S.sif_k_rope(rope, S.rope_args(a, b, rows, h, d, seq=rows, first=p))
    S.sif_k_rope(rope, S.rope_args(dy, out[2], rows, h, d, seq=rows, first=p, inverse=True))
    y0, y1, dx = (o.double().cpu() for o in out)
    dy, along = dy.double().cpu(), (plus.double() - minus.double()).cpu()
    slope, says = (dy * (y0 - y1)).sum(), (dx * along).sum()
    # each of the three results is rounded once, and turned elements are fp32 sums of two
    bound = (dy.abs() * (y0.abs() + y1.abs()) * HALF).sum() + (dx.abs() * along.abs() * HALF).sum() + 2.0 ** -20 * 1.5 * 2 * (dy.abs().max() * along.abs()).sum()
    assert abs(float(slope - says)) <= float(bound) and abs(float(says)) > 0
    assert abs(float(slope - says)) <= 2e-3 * float((dy.norm() * along.norm()))      # (and in the norm: half a step is 1.7e-3 together)


def test_rows_past_32_bits():
    ld, rows = 1 << 26, 40
    wide = torch.zeros(rows, ld, dtype=torch.bfloat16, device=DEV)      # 5 GB
    q = _x(9, rows, 128)
    wide[:, 256:384] = q.to(DEV)
    S.sif_k_rope(S.rope_plan(128), S.rope_args(wide[:, 256:384], wide[:, 512:640], rows, 1, 128, seq=rows))
    val, off = turned(q.double().view(rows, 1, 128), torch.arange(rows), frequencies(128), False)
    assert torch.all((wide[:, 512:640].cpu().double() - val[:, 0]).abs() <= HALF * val[:, 0].abs() + 2 * off[:, 0] + 1e-38)
    assert torch.equal(wide[:, 256:384].cpu(), q) and not wide[:, 640:768].any() and not wide[:, :256].any()


def test_on_another_stream_and_in_a_graph():
    rope, q = S.rope_plan(64), _x(10, 100, 256)
    x, out, back = q.to(DEV), torch.empty(100, 256, dtype=torch.bfloat16, device=DEV), torch.empty(100, 256, dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(100, dtype=torch.int32, device=DEV)
    fa, ba = S.rope_args(x, out, 100, 4, 64, positions=pos), S.rope_args(out, back, 100, 4, 64, positions=pos, inverse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.sif_k_rope(rope, fa, stream=side)
        S.sif_k_rope(rope, ba, stream=side)
    side.synchronize()
    want, want_back = out.clone(), back.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.sif_k_rope(rope, fa, stream=torch.cuda.current_stream())
        S.sif_k_rope(rope, ba, stream=torch.cuda.current_stream())
    rope = None                                      # (the launches hold the table)
    for _ in range(3):
        out.zero_()
        back.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(back, want_back)
    x.copy_(_x(11, 100, 256).to(DEV))
    pos += 5
    graph.replay()
    _check(torch.cat([out, torch.full((100, 8), 7.0, dtype=torch.bfloat16, device=DEV)], 1), x.cpu(), torch.arange(100) + 5, frequencies(64), 4, 64, False, 1.0, False, "new inputs")
