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
