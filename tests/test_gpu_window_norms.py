"""Attention with a sliding window and sinks, forward and backward, by the norms of what results are off, against those that the kernels'
roundings make."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import attn_rounding
from attn_reference import heads_attention, visible

if torch.cuda.is_available():
    from test_gpu_window_attention import Run, _inputs


@pytest.mark.parametrize("lens,heads,kv_heads,d,window,sinks", [
    ([16, 16, 40, 611], 8, 8, 64, 0, 0),
    ([16, 16, 40, 611], 8, 2, 64, 4096, 4),       # a window that no sequence reaches
    ([611, 40, 16, 16], 8, 4, 128, 0, 0),
    ([16, 40, 611, 16], 8, 8, 128, 300, 4),
])
def test_short_sequences_beside_a_long_one(lens, heads, kv_heads, d, window, sinks):
    """Gradients of a sequence are as near as they are where it stands alone, whatever else the call holds."""
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    q, k, v, do = _inputs(71 + d + window, starts[-1], starts[-1], heads, kv_heads, d)
    run = Run(q, k, v, do, heads, kv_heads, d, len(lens), max(lens), max(lens), window, sinks, starts=starts)
    run.forward()
    run.backward()
    got = run.results()
    for i, m in enumerate(lens):
        r = slice(starts[i], starts[i] + m)
        x, seen = [t[r].double() for t in (q, k, v)], visible(m, m, window, sinks)
        stored = got["o"][r].double().cpu()
        val, _ = heads_attention(*x, heads, kv_heads, d, seen, 1 / math.sqrt(d), do[r].double())
        model = attn_rounding.heads(*x, heads, kv_heads, d, seen, 1 / math.sqrt(d), do[r].double(), o=stored if m > 256 else None)
        attn_rounding.assert_near({n: y[r] for n, y in got.items() if n != "lse"}, val, model, {}, (i, m))
        if m > 256:                                # the first rows of a long one see few keys too
            model = attn_rounding.heads(*x, heads, kv_heads, d, seen, 1 / math.sqrt(d), do[r].double())
            attn_rounding.assert_near({"dq": got["dq"][r]}, val, {"dq": model["dq"]}, {"dq": slice(0, 64)}, (i, m, "its first rows"))


@pytest.mark.parametrize("batch,sq,sk,heads,kv_heads,d,window,sinks", attn_rounding.CASES)
def test_results_are_as_near_as_their_roundings_let_them(batch, sq, sk, heads, kv_heads, d, window, sinks):
    """All results together, and the sinks' gradients, which are put together from pieces, by themselves."""
    q, k, v, do = attn_rounding.inputs(sq + 7 * sk + window, batch * sq, batch * sk, heads, kv_heads, d)
    run = Run(q, k, v, do, heads, kv_heads, d, batch, sq, sk, window, sinks, pad=8)
    run.forward()
    run.backward()
    got, seen = run.results(), visible(sq, sk, window, sinks)
    few = int(seen.sum(1).max()) <= 256            # (there the row term is taken from the scores)
    for b in range(batch):
        rq, rk = slice(b * sq, (b + 1) * sq), slice(b * sk, (b + 1) * sk)
        x = (q[rq].double(), k[rk].double(), v[rk].double(), heads, kv_heads, d, seen, 1 / math.sqrt(d), do[rq].double())
        val, _ = heads_attention(*x)
        mine = {n: got[n][rq if n in ("o", "dq") else rk] for n in ("o", "dq", "dk", "dv")}
        model = attn_rounding.heads(*x, o=None if few else mine["o"].double().cpu())
        attn_rounding.assert_near(mine, val, model, {}, b)
        if sinks:
            attn_rounding.assert_near(mine, val, {n: model[n] for n in ("dk", "dv")}, dict.fromkeys(("dk", "dv"), slice(0, sinks)), (b, "sinks"))


@pytest.mark.parametrize("sq,sk,heads,kv_heads,d,window,sinks", [(96, 96, 2, 1, 64, 24, 2), (80, 130, 4, 2, 128, 40, 5)])
def test_gradients_are_the_slopes_of_the_forward_pass(sq, sk, heads, kv_heads, d, window, sinks):
    """<o, do> from the operator's own forward pass, a step up and a step down the gradient of each input, against its gradients."""
    q, k, v, do = attn_rounding.inputs(33, sq, sk, heads, kv_heads, d)
    seen, scale, x = visible(sq, sk, window, sinks), 1 / math.sqrt(d), [q, k, v]
    run = Run(q, k, v, do, heads, kv_heads, d, 1, sq, sk, window, sinks)
    run.forward()
    run.backward()
    got = run.results()
    exact = lambda y, *grad: heads_attention(*(t.double() for t in y), heads, kv_heads, d, seen, scale, *grad)      # noqa: E731
    val, tol = exact(x, do.double())
    model = attn_rounding.heads(*(t.double() for t in x), heads, kv_heads, d, seen, scale, do.double())
    for of, name in enumerate(("dq", "dk", "dv")):
        up, loss, true = val[name] / val[name].norm(), [], []
        ends = [(x[of].double() + sign * 2.0 * up).to(torch.bfloat16) for sign in (1.0, -1.0)]
        step = ends[0].double() - ends[1].double()
        for end in ends:
            y = list(x)
            y[of] = end
            there = Run(*y, do, heads, kv_heads, d, 1, sq, sk, window, sinks)
            there.forward()
            loss.append(float((there.results()["o"].double().cpu() * do.double()).sum()))
            true.append(float((exact(y)[0]["o"] * do.double()).sum()))
        slope = float((val[name] * step).sum())
        bent = abs(true[0] - true[1] - slope)      # what the differences leave of higher orders
        # three times the root mean square of what rounding adds to the two sums (an error within +-t is t / sqrt(3) there), and the gradient's norm
        noise = 3.0 * math.sqrt(2.0 / 3.0) * float((do.double() * tol["o"]).norm())
        bound = bent + noise + attn_rounding.GRADIENTS * float((model[name] - val[name]).norm() * step.norm())
        assert bound <= 0.1 * slope, (name, bent, noise, slope)
        assert abs(loss[0] - loss[1] - float((got[name].double().cpu() * step).sum())) <= bound, name
