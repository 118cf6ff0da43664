"""Attention with a sliding window and sinks, forward and backward, against the formulas in 64 bits, element by element."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_reference import assert_within, heads_attention, visible

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV


def _inputs(seed, rq, rk, heads, kv_heads, d, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda n, w, x: (x * torch.randn(n, w, generator=g)).to(torch.bfloat16)      # noqa: E731
    return r(rq, heads * d, spread), r(rk, kv_heads * d, spread), r(rk, kv_heads * d, 1.0), r(rq, heads * d, 1.0)


class Run:
    """The operator on copies of the inputs in wider buffers: rows of other leading dimensions, canaries around the results."""

    def __init__(self, q, k, v, do, heads, kv_heads, d, batch, sq, sk, window, sinks, pad=0, starts=None, lse=True, scale=0.0, stream=None):
        def wide(x):
            if x is None:
                return None
            w = torch.full((x.shape[0], x.shape[1] + pad), math.nan, dtype=torch.bfloat16, device=DEV)
            w[:, :x.shape[1]] = x.to(DEV)
            return w
        self.q, self.k, self.v, self.do = (wide(x) for x in (q, k, v, do))
        self.o, self.dq, self.dk, self.dv = (torch.full_like(x, 7.0) if x is not None else None for x in (self.q, self.q, self.k, self.k))
        self.lse = torch.full((heads, q.shape[0]), 7.0, device=DEV) if lse else None
        self.starts = None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
        self.args = S.window_attn_args(self.q, self.k, self.v, self.o, heads, kv_heads, d, batch, sq, sk, window, sinks, lse=self.lse, starts=self.starts,
                                       rows=q.shape[0] if starts is not None else 0, scale=scale, d_o=self.do, dq=self.dq, dk=self.dk, dv=self.dv)
        self.wq, self.wk, self.stream = heads * d, kv_heads * d, stream
        if do is not None:
            n = S.sif_window_attn_bwd_workspace_bytes(self.args)
            self.work = torch.empty(n, dtype=torch.uint8, device=DEV)
            S.set_workspace(self.args, self.work, n)
        torch.cuda.synchronize()

    def forward(self):
        S.sif_k_window_attn_fwd(self.args, stream=self.stream)

    def backward(self):
        S.sif_k_window_attn_bwd(self.args, stream=self.stream)

    def results(self):
        torch.cuda.synchronize()
        got = {"o": self.o[:, :self.wq], "dq": self.dq[:, :self.wq], "dk": self.dk[:, :self.wk], "dv": self.dv[:, :self.wk]}
        if self.lse is not None:
            got["lse"] = self.lse
        for t, w in ((self.o, self.wq), (self.dq, self.wq), (self.dk, self.wk), (self.dv, self.wk)):
            assert bool((t[:, w:] == 7.0).all()), "columns behind the rows were written"
        return got


def _check(run, q, k, v, do, heads, kv_heads, d, parts, window, sinks, backward=True, scale=None):
    """parts: (first query row, queries, first key row, keys) of each sequence."""
    got = run.results()
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    exact = run.args.seq_k <= 256 or 0 < window <= 256 - sinks
    for i, (a, m, b, n) in enumerate(parts):
        rq, rk = slice(a, a + m), slice(b, b + n)
        val, tol = heads_attention(q[rq].double(), k[rk].double(), v[rk].double(), heads, kv_heads, d, visible(m, n, window, sinks), scale,
                                   do[rq].double() if backward else None, exact)
        for name in val:
            if name == "lse":
                if run.lse is not None:
                    assert_within(got["lse"][:, rq], val["lse"], tol["lse"], (i, "lse"))
            else:
                assert_within(got[name][rk if name in ("dk", "dv") else rq], val[name], tol[name], (i, name))


CASES = [
    # batch, queries, keys, heads, kv heads, d, window, sinks
    (1, 1, 1, 1, 1, 64, 1, 0),
    (1, 1, 1, 4, 1, 128, 0, 0),
    (2, 1, 300, 4, 2, 64, 40, 3),                 # single rows behind a cache
    (1, 33, 33, 2, 2, 64, 1, 0),                  # every row sees itself alone
    (1, 33, 33, 2, 2, 128, 1, 1),
    (2, 64, 64, 4, 2, 64, 16, 2),
    (1, 129, 129, 3, 1, 64, 31, 5),               # a group of three query heads
    (1, 129, 129, 3, 3, 128, 32, 128),            # as many sinks as there can be
    (1, 257, 257, 8, 2, 128, 33, 4),
    (1, 257, 257, 8, 1, 64, 63, 4),               # eight query heads to a key head
    (1, 300, 300, 2, 1, 128, 64, 0),
    (1, 300, 300, 2, 1, 64, 0, 0),                # no window: causal
    (1, 300, 300, 2, 2, 128, 0, 9),               # no window: sinks mean nothing
    (1, 300, 300, 4, 4, 64, 1000, 4),             # a window past the sequence
    (1, 100, 517, 4, 1, 128, 130, 7),             # a prompt's next piece
    (1, 100, 517, 4, 1, 64, 600, 7),
    (2, 70, 31, 4, 2, 64, 12, 2),                 # more queries than keys: the first rows see nothing
    (1, 200, 31, 2, 2, 128, 0, 0),
    (1, 700, 700, 6, 2, 64, 200, 70),             # sinks of more than one piece of 32
    (1, 700, 700, 4, 4, 128, 129, 33),
    (1, 1500, 1500, 4, 1, 128, 256, 4),
    (3, 391, 391, 4, 2, 64, 100, 100),
]


@pytest.mark.parametrize("batch,sq,sk,heads,kv_heads,d,window,sinks", CASES)
def test_forward_and_backward(batch, sq, sk, heads, kv_heads, d, window, sinks):
    q, k, v, do = _inputs(sq + 7 * sk + window, batch * sq, batch * sk, heads, kv_heads, d)
    run = Run(q, k, v, do, heads, kv_heads, d, batch, sq, sk, window, sinks, pad=8)
    run.forward()
    run.backward()
    _check(run, q, k, v, do, heads, kv_heads, d, [(b * sq, sq, b * sk, sk) for b in range(batch)], window, sinks)


@pytest.mark.parametrize("d,window,sinks", [(64, 20, 3), (128, 50, 40), (64, 0, 0)])
def test_packed_sequences(d, window, sinks):
    """Sequences of unequal length back to back, empty ones among them, rows in front, between and behind that belong to none."""
    heads, kv_heads, lens, first = 4, 2, [0, 1, 130, 0, 64, 257], 5
    starts = [first + sum(lens[:i]) for i in range(len(lens) + 1)]
    rows = starts[-1] + 9
    q, k, v, do = _inputs(d + window, rows, rows, heads, kv_heads, d)
    for x in (q, k, v, do):                        # what belongs to no sequence may hold anything
        x[:first] = math.nan
        x[starts[-1]:] = math.nan
    run = Run(q, k, v, do, heads, kv_heads, d, len(lens), 257, 257, window, sinks, starts=starts)
    run.forward()
    run.backward()
    got = run.results()
    _check(run, q, k, v, do, heads, kv_heads, d, [(starts[i], m, starts[i], m) for i, m in enumerate(lens) if m], window, sinks)
    for name in ("o", "dq", "dk", "dv"):
        assert bool((got[name][:first] == 7.0).all()) and bool((got[name][starts[-1]:] == 7.0).all()), name
    assert bool((got["lse"][:, :first] == 7.0).all()) and bool((got["lse"][:, starts[-1]:] == 7.0).all())


def test_a_packed_sequence_longer_than_announced_is_cut():
    heads, kv_heads, d, starts = 2, 1, 64, [0, 200, 230]
    q, k, v, do = _inputs(3, 230, 230, heads, kv_heads, d)
    run = Run(q, k, v, do, heads, kv_heads, d, 2, 150, 150, 40, 2, starts=starts)
    run.forward()
    run.backward()
    got = run.results()
    _check(run, q, k, v, do, heads, kv_heads, d, [(0, 150, 0, 150), (200, 30, 200, 30)], 40, 2)
    for name in ("o", "dq", "dk", "dv"):
        assert bool((got[name][150:200] == 7.0).all()), name


def test_keys_and_rows_that_nobody_sees_have_no_influence():
    """Keys in front of every window and behind the sinks hold NaN; rows that see nothing hold NaN in q and do."""
    heads, kv_heads, d, sq, sk, window, sinks = 4, 2, 128, 60, 400, 70, 3
    q, k, v, do = _inputs(9, sq, sk, heads, kv_heads, d)
    unseen = slice(sinks, sk - sq - window + 1)
    clean = [x.clone() for x in (k, v)]
    k[unseen] = math.nan
    v[unseen] = math.inf
    run = Run(q, k, v, do, heads, kv_heads, d, 1, sq, sk, window, sinks)
    run.forward()
    run.backward()
    _check(run, q, *clean, do, heads, kv_heads, d, [(0, sq, 0, sk)], window, sinks)
    sq, sk = 90, 40
    q, k, v, do = _inputs(10, sq, sk, heads, kv_heads, d)
    clean = [x.clone() for x in (q, do)]
    q[:sq - sk], do[:sq - sk] = math.nan, math.nan
    run = Run(q, k, v, do, heads, kv_heads, d, 1, sq, sk, 8, 2)
    run.forward()
    run.backward()
    _check(run, clean[0], k, v, clean[1], heads, kv_heads, d, [(0, sq, 0, sk)], 8, 2)


@pytest.mark.parametrize("d", [64, 128])
def test_large_scores_and_a_rising_maximum(d):
    """Scores up to some hundred, growing along the keys, so that the running maximum has to follow; a scale of the caller's own."""
    heads, kv_heads, s = 2, 1, 400
    q, k, v, do = _inputs(21, s, s, heads, kv_heads, d, spread=2.0)
    k = (k.float() * torch.linspace(0.1, 3.0, s)[:, None]).to(torch.bfloat16)
    run = Run(q, k, v, do, heads, kv_heads, d, 1, s, s, 300, 4, scale=0.3)
    run.forward()
    run.backward()
    _check(run, q, k, v, do, heads, kv_heads, d, [(0, s, 0, s)], 300, 4, scale=float(torch.tensor(0.3)))


def test_rows_past_31_bits_of_bytes():
    """A leading dimension that takes the last rows beyond 4 GiB."""
    heads, kv_heads, d, s = 1, 1, 64, 300
    q, k, v, do = _inputs(5, s, s, heads, kv_heads, d)
    ld = 8 * 1024 * 1024
    wide = torch.zeros(s, ld, dtype=torch.bfloat16, device=DEV)      # 5 GB; q, k and v lie side by side
    for i, x in enumerate((q, k, v)):
        wide[:, i * 64:i * 64 + 64] = x.to(DEV)
    o, lse = torch.empty(s, 64, dtype=torch.bfloat16, device=DEV), torch.empty(1, s, device=DEV)
    a = S.window_attn_args(wide, wide[:, 64:], wide[:, 128:], o, heads, kv_heads, d, 1, s, s, 50, 2, lse=lse)
    S.sif_k_window_attn_fwd(a)
    torch.cuda.synchronize()
    val, tol = heads_attention(q.double(), k.double(), v.double(), 1, 1, 64, visible(s, s, 50, 2), 0.125)
    assert_within(o, val["o"], tol["o"], "o")
    assert_within(lse, val["lse"], tol["lse"], "lse")


def test_gradients_against_differences():
    """The gradient of <o, do> along a direction, from forward passes a step apart (on inputs that bf16 holds exactly)."""
    heads, kv_heads, d, s, window, sinks = 2, 1, 64, 96, 24, 2
    q, k, v, do = _inputs(33, s, s, heads, kv_heads, d)
    run = Run(q, k, v, do, heads, kv_heads, d, 1, s, s, window, sinks)
    run.forward()
    run.backward()
    got = run.results()
    g = torch.Generator().manual_seed(4)
    for name, of in (("dq", 0), ("dk", 1), ("dv", 2)):
        x = [t.double() for t in (q, k, v)]
        direction = torch.randn(x[of].shape, generator=g, dtype=torch.float64)
        loss = []
        for sign in (1.0, -1.0):
            y = list(x)
            y[of] = x[of] + sign * 1e-4 * direction
            val, _ = heads_attention(*y, heads, kv_heads, d, visible(s, s, window, sinks), 0.125)
            loss.append(float((val["o"] * do.double()).sum()))
        slope = (loss[0] - loss[1]) / 2e-4
        _, tol = heads_attention(*x, heads, kv_heads, d, visible(s, s, window, sinks), 0.125, do.double())
        mine = got[name].double().cpu()
        assert abs(float((mine * direction).sum()) - slope) <= float((tol[name] * direction.abs()).sum()) + 1e-5 * abs(slope), name


def test_without_lse_forward_is_the_same_and_runs_are_alike_bit_for_bit():
    heads, kv_heads, d, s = 8, 2, 128, 600
    q, k, v, do = _inputs(12, s, s, heads, kv_heads, d)
    a, b = (Run(q, k, v, do, heads, kv_heads, d, 1, s, s, 150, 4, lse=x) for x in (True, False))
    a.forward()
    b.forward()
    a.backward()
    first = {x: y.clone() for x, y in a.results().items()}
    assert torch.equal(first["o"], b.results()["o"])
    a.forward()
    a.backward()
    for x, y in a.results().items():
        assert torch.equal(first[x], y), x


def test_two_streams_at_once_and_a_graph():
    """Two calls side by side on streams of their own, with workspaces of their own; then both passes captured and replayed with other inputs."""
    shape = dict(heads=4, kv_heads=2, d=64, batch=1, sq=500, sk=500, window=90, sinks=4)
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = [_inputs(40 + i, 500, 500, 4, 2, 64) for i in range(3)]
    runs = [Run(*sets[i], **shape, stream=streams[i]) for i in range(2)]
    for _ in range(3):
        for r in runs:
            r.forward()
            r.backward()
    for i, r in enumerate(runs):
        _check(r, *sets[i], 4, 2, 64, [(0, 500, 0, 500)], 90, 4)
    r = Run(*sets[0], **shape)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        r.stream = torch.cuda.current_stream()
        r.forward()
        r.backward()
    for i in (1, 2, 0):
        for into, x in zip((r.q, r.k, r.v, r.do), sets[i]):
            into.copy_(x.to(DEV))
        torch.cuda.synchronize()
        graph.replay()
        _check(r, *sets[i], 4, 2, 64, [(0, 500, 0, 500)], 90, 4)
