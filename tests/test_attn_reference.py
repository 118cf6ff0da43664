"""The references that the attention operators are tested against: the formulas in 64 bits against autograd, and the bounds on norms against
planted mistakes."""
import math

import pytest
import torch

import attn_rounding
from attn_reference import heads_attention, visible


@pytest.mark.parametrize("sq,sk,heads,kv_heads,d,window,sinks", [(33, 33, 2, 2, 64, 0, 0), (60, 60, 4, 2, 64, 9, 3), (20, 75, 4, 1, 64, 30, 4), (50, 31, 2, 1, 64, 12, 2)])
def test_the_formulas_are_those_of_autograd(sq, sk, heads, kv_heads, d, window, sinks):
    q, k, v, do = (x.double() for x in attn_rounding.inputs(1, sq, sk, heads, kv_heads, d))
    seen = visible(sq, sk, window, sinks)
    val, _ = heads_attention(q, k, v, heads, kv_heads, d, seen, 0.125, do)
    x = [t.clone().requires_grad_(True) for t in (q, k, v)]
    some = seen.any(1)                             # (rows that see nothing have zeros, and autograd of their softmax has none to give)
    group, out = heads // kv_heads, []
    for h in range(heads):
        cq, ck = slice(h * d, h * d + d), slice(h // group * d, h // group * d + d)
        s = (x[0][some][:, cq] @ x[1][:, ck].t() * 0.125).masked_fill(~seen[some], -math.inf)
        out.append(torch.softmax(s, 1) @ x[2][:, ck])
    o = torch.cat(out, 1)
    grads = torch.autograd.grad(o, x, do[some])
    assert torch.allclose(val["o"][some], o, rtol=1e-11, atol=1e-11) and not val["o"][~some].any()
    for name, g in zip(("dq", "dk", "dv"), grads):
        assert torch.allclose(val[name], g, rtol=1e-10, atol=1e-10), name


def _far(sq, sk, window):
    """First row that sees nothing of the first 128 keys but the sinks."""
    return max(min(127, sk - 1) + window - (sk - sq), 0) if window else sq


@pytest.mark.parametrize("batch,sq,sk,heads,kv_heads,d,window,sinks", attn_rounding.CASES)
def test_planted_mistakes_pass_the_bounds(batch, sq, sk, heads, kv_heads, d, window, sinks):
    q, k, v, do = (x.double() for x in attn_rounding.inputs(sq + 7 * sk + window, sq, sk, heads, kv_heads, d))
    x = (q, k, v, heads, kv_heads, d, visible(sq, sk, window, sinks), 1 / math.sqrt(d), do)
    val, _ = heads_attention(*x)
    model = attn_rounding.heads(*x)
    stored = attn_rounding.heads(*x, o=model["o"])
    attn_rounding.assert_near(model, val, stored, {}, "none")

    def caught(got, rows):
        with pytest.raises(AssertionError):
            attn_rounding.assert_near(got, val, {n: stored[n] for n in got}, rows, "planted")
    wrong = attn_rounding.heads(*x, change="no row term")
    for name in ("dq", "dk"):
        caught({name: wrong[name]}, {})
    for name in val:
        if name != "lse":
            caught({name: torch.zeros_like(val[name])}, {})
            caught({name: -model[name]}, {})
    far = _far(sq, sk, window)
    if sinks and far < sq:
        row, key = torch.arange(sq)[:, None], torch.arange(sk)[None, :]
        of_sinks = (row >= far) & (key < sinks)
        near = {"dk": slice(0, sinks)}
        caught({"dk": attn_rounding.heads(*x, lost=lambda h: of_sinks)["dk"]}, near)
        piece = of_sinks & (row < far + 256)       # eight times 32 rows of one query head
        caught({"dk": attn_rounding.heads(*x, lost=lambda h: piece & (h == 0))["dk"]}, near)
        assert far + 32 < sq
