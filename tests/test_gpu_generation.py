"""Rotations, the paged cache in 4 bits, attention over it and the choice of tokens as a generating program runs them together, and rotations around attention as a training step does."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_reference import assert_within, attention, heads_attention, visible
from rows_reference import HALF, Rows, frequencies, sample, turned

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV


def _x(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


class Step:
    """One layer of a decoder that generates: product for q, k and v, rotation and cache, attention, logits, token.  Buffers and argument structures are set up once."""

    def __init__(self, rows, heads, vocab, seed, n):
        h, d, self.dm = rows.h, rows.d, 128
        self.rows, self.heads, self.vocab, self.n = rows, heads, vocab, n
        cache = self.cache = rows.on(S, DEV)
        w = (heads + 2 * h) * d
        self.wqkv, self.embed, self.head = (_x(seed + i, *s).mul(f).to(DEV) for i, (s, f) in enumerate((((w, self.dm), 0.3), ((vocab, self.dm), 1.0), ((vocab, heads * d), 0.2))))
        bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)      # noqa: E731
        self.x, self.qkv, self.o, self.logits = bf(n, self.dm), bf(n, w), bf(n, heads * d), torch.zeros(n, vocab, device=DEV)
        self.token, self.logprob, self.random = torch.arange(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        self.seqs = torch.arange(n, dtype=torch.int32, device=DEV)
        size = S.sif_kv_workspace_bytes(cache)
        self.work = torch.zeros(size, dtype=torch.uint8, device=DEV)
        self.rope = S.rope_plan(d, base=500.0)
        q, k, v = self.qkv[:, :heads * d], self.qkv[:, heads * d:(heads + h) * d], self.qkv[:, (heads + h) * d:]
        self.append = S.kv_append_args(k, v, n, seqs=self.seqs, q=q, heads=heads)
        self.decode = S.attn_decode_args(q, self.o, n, heads, seqs=self.seqs)
        size = S.sif_attn_decode_workspace_bytes(cache, self.decode)
        self.scratch = torch.zeros(size, dtype=torch.uint8, device=DEV)
        S.set_workspace(self.decode, self.scratch, size)
        self.choose = S.sample_args(self.logits, self.token, n, vocab, random=self.random, temperature=0.9, top_k=40, top_p=0.95, min_p=0.01, logprob=self.logprob)

    def run(self, stream=None):
        torch.index_select(self.embed, 0, self.token.long(), out=self.x)
        self._product(self.x, self.wqkv, self.qkv, 0, stream)
        S.sif_k_kv_extend(self.cache, self.seqs, None, self.n, self.work, self.work.numel(), stream=stream)
        S.sif_k_kv_append(self.cache, self.rope, self.append, stream=stream)
        S.sif_k_attn_decode(self.cache, self.decode, stream=stream)
        self._product(self.o, self.head, self.logits, S.SIF_EPI_OUT_F32, stream)
        S.sif_k_sample(self.choose, stream=stream)

    def _product(self, a, b, c, epilogue, stream):
        g = S.sif_gemm_args()
        g.struct_size, g.epilogue = S.C.sizeof(S.sif_gemm_args), epilogue
        g.m, g.n, g.k, g.lda, g.ldb, g.ldc = a.shape[0], b.shape[0], a.shape[1], a.stride(0), b.stride(0), c.stride(0)
        g.batch_outer = g.batch_inner = 1
        g.alpha, g.a_dev, g.b_dev, g.c_dev = 1.0, a.data_ptr(), b.data_ptr(), c.data_ptr()
        S.check(S.lib.sif_k_gemm_bf16(S.C.byref(g), S.stream_ptr(stream)))


def _rows(seed):
    return Rows("e2m1", [31, 5, 64, 100], 16, 2, 64, layers=1, seed=seed, spare=20, wider=4)


def test_tokens_one_after_the_other():
    """Every product of a step from what the step before it left, each against its definition."""
    rows, heads, vocab = _rows(1), 6, 304
    s = Step(rows, heads, vocab, 10, 4)
    d, h, f, seen_tokens = 64, 2, frequencies(64, base=500.0), []
    for t in range(4):
        s.random.copy_(torch.rand(4, generator=torch.Generator().manual_seed(t)).to(DEV))
        s.run()
        torch.cuda.synchronize()
        # the operations on pages as they define them
        taken = rows.t["table"].cpu().tolist()
        for i in range(4):
            rows.lens[i] += 1
            rows.table[i] = taken[i]
        assert rows.t["lengths"].cpu().tolist() == rows.lens
        x = s.x.cpu().double()
        qkv = x @ s.wqkv.cpu().double().t()
        got = s.qkv.cpu().double()
        # (k and v as the product left them: the step turns q in its place)
        assert torch.all((got - qkv)[:, heads * d:].abs() <= HALF * qkv[:, heads * d:].abs() + 2.0 ** -16 * (x.abs() @ s.wqkv.cpu().double().abs().t())[:, heads * d:])
        for i in range(4):
            pos = torch.tensor([rows.lens[i] - 1])
            val, off = turned(qkv[i, :heads * d].view(1, heads, d), pos, f, False)
            spread = torch.sqrt((qkv[i, :heads * d] ** 2).view(1, heads, 2, d // 2).sum(2, keepdim=True)).expand(1, heads, 2, d // 2).reshape(1, heads, d)
            assert torch.all((got[i, :heads * d].view(1, heads, d) - val).abs() <= HALF * val.abs() + off + 2 * HALF * spread + 1e-3)      # rounded before it is turned, too
            val, _ = turned(got[i, heads * d:(heads + h) * d].view(1, h, d), pos, f, False)
            rows.put("k", 0, i, int(pos), val[0])
            rows.put("v", 0, i, int(pos), got[i, (heads + h) * d:].view(h, d))
        rows.check()
        for i in range(4):
            m = rows.lens[i]
            k, v = (torch.stack([rows.get(z, 0, i, j) for j in range(m)]) for z in "kv")
            for g in range(h):
                c = slice(g * 3 * d, (g + 1) * 3 * d)
                val, tol = attention(got[i, c].view(3, d), k[:, g], v[:, g], torch.ones(3, m, dtype=torch.bool), 1 / math.sqrt(d))
                assert_within(s.o[i, c].view(3, d), val["o"], tol["o"], (t, i, g))
            token, logprob, _ = sample(s.logits[i].cpu().double().numpy(), float(s.random[i]), float(torch.tensor(0.9)), 40, float(torch.tensor(0.95)), float(torch.tensor(0.01)))
            assert int(s.token[i]) == token and abs(float(s.logprob[i]) - logprob) <= 2.0 ** -23 * abs(logprob) + 1e-9
            seen_tokens.append(token)
    assert len(set(seen_tokens)) > 4


def test_a_captured_step_goes_on_by_itself():
    """One graph for a whole step: replays lengthen the sequences, take pages, write, attend and choose, as the same calls do eagerly."""
    u = [torch.rand(4, generator=torch.Generator().manual_seed(t)).to(DEV) for t in range(12)]
    eager, rows = Step(_rows(2), 6, 304, 20, 4), None
    want = []
    for t in range(12):
        eager.random.copy_(u[t])
        eager.run()
        want.append((eager.token.clone(), eager.logprob.clone(), eager.o.clone()))
    rows = _rows(2)
    s = Step(rows, 6, 304, 20, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run(side)                                        # (the product's first launch sets up what it keeps)
    side.synchronize()
    for name in ("k", "v", "table", "lengths", "refs"):
        fresh = _rows(2)
        fresh.on(S, DEV)
        rows.t[name].copy_(fresh.t[name])
    s.token.copy_(torch.arange(4, dtype=torch.int32, device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run(side)
    for t in range(12):
        s.random.copy_(u[t])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((s.token, s.logprob, s.o), want[t]):
            assert torch.equal(a, b), t
    for name in ("k", "v", "table", "lengths", "refs"):
        assert torch.equal(rows.t[name], eager.rows.t[name]), name


def test_two_programs_at_once():
    """Steps of two programs under way at the same time, on streams, caches and workspaces of their own."""
    def start(seed):
        return Step(_rows(seed), 6, 304, 20 + seed, 4)

    def numbers(seed):
        return [torch.rand(4, generator=torch.Generator().manual_seed(100 * seed + t)).to(DEV) for t in range(10)]
    want = {}
    for seed in (3, 4):
        s = start(seed)
        for u in numbers(seed):
            s.random.copy_(u)
            s.run()
        want[seed] = [x.clone() for x in (s.token, s.logprob, s.o, s.rows.t["k"], s.rows.t["v"], s.rows.t["lengths"], s.rows.t["table"])]
    both, streams = [start(3), start(4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    given = [numbers(3), numbers(4)]
    torch.cuda.synchronize()
    for t in range(10):
        for s, stream, u in zip(both, streams, given):
            with torch.cuda.stream(stream):
                s.random.copy_(u[t])
                s.run(stream)
    torch.cuda.synchronize()
    for seed, s in zip((3, 4), both):
        for a, b in zip((s.token, s.logprob, s.o, s.rows.t["k"], s.rows.t["v"], s.rows.t["lengths"], s.rows.t["table"]), want[seed]):
            assert torch.equal(a, b), seed


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "e2m1"])
def test_a_prompt_in_pieces(dtype):
    """The next piece of a prompt attends to what the cache holds of the earlier ones: written, read back as rows, windowed attention over them."""
    heads, h, d, first, second = 4, 2, 64, 70, 45
    rows = Rows(dtype, [first + second], 16, h, d, layers=1, seed=3)
    cache = rows.on(S, DEV)
    q, k, v = _x(1, first + second, heads * d).to(DEV), _x(2, first + second, h * d).to(DEV), _x(3, first + second, h * d).to(DEV)
    one = torch.tensor([0, first + second], dtype=torch.int32, device=DEV)
    out = torch.empty_like(q)
    S.sif_k_kv_append(cache, S.rope_plan(64), S.kv_append_args(k, v, 1, rows=first + second, starts=one, q=q, q_out=out, heads=heads))
    kr, vr = torch.empty_like(k), torch.empty_like(v)
    S.sif_k_kv_read(cache, 0, kr, vr, None, 1, starts=one, rows=first + second)
    o, lse = torch.empty(second, heads * d, dtype=torch.bfloat16, device=DEV), torch.empty(heads, second, device=DEV)
    S.sif_k_window_attn_fwd(S.window_attn_args(out[first:], kr, vr, o, heads, h, d, 1, second, first + second, 0, 0, lse=lse))
    val, tol = heads_attention(out[first:].cpu().double(), kr.cpu().double(), vr.cpu().double(), heads, h, d, visible(second, first + second, 0, 0), 1 / math.sqrt(d))
    assert_within(o, val["o"], tol["o"], "o")
    assert_within(lse, val["lse"], tol["lse"], "lse")
    # the last row is what decoding over the cache says of it
    last, scratch = torch.empty(1, heads * d, dtype=torch.bfloat16, device=DEV), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    a = S.attn_decode_args(out[-1:], last, 1, heads)
    S.set_workspace(a, scratch, 1 << 20)
    S.sif_k_attn_decode(cache, a)
    # (e4m3 values times their scales are rounded to bf16 on their way back: one more half step of keys, through the scores, and of values)
    more = 0.0 if dtype != "e4m3" else HALF * (1.0 + 2.0 * float((out[-1].cpu().double().abs().view(heads, d).sum(1) / math.sqrt(d)).max()) * float(kr.abs().max()))
    assert torch.all((last.cpu().double()[0] - val["o"][-1]).abs() <= tol["o"][-1] + more * float(vr.abs().max()))


def test_a_training_step_turns_queries_and_keys():
    """Rotation, attention, its gradients and the rotation back: each from what the one before it left, against its formulas."""
    heads, h, d, rot, n = 4, 2, 64, 32, 130
    f, rope = frequencies(rot), S.rope_plan(rot)
    q, k, v, do = _x(4, n, heads * d), _x(5, n, h * d), _x(6, n, h * d), _x(7, n, heads * d)
    q, k, v, do = (x.to(DEV) for x in (q, k, v, do))
    tq, tk, o, lse = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty(heads, n, device=DEV)
    dq, dk, dv, gq, gk = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    fwd, bwd = S.rope_args(q, tq, n, heads, d, k=k, k_out=tk, kv_heads=h, seq=n), S.rope_args(dq, gq, n, heads, d, k=dk, k_out=gk, kv_heads=h, seq=n, inverse=True)
    a = S.window_attn_args(tq, tk, v, o, heads, h, d, 1, n, n, 0, 0, lse=lse, d_o=do, dq=dq, dk=dk, dv=dv)
    size = S.sif_window_attn_bwd_workspace_bytes(a)
    work = torch.empty(size, dtype=torch.uint8, device=DEV)
    S.set_workspace(a, work, size)

    def step(stream=None):
        S.sif_k_rope(rope, fwd, stream=stream)
        S.sif_k_window_attn_fwd(a, stream=stream)
        S.sif_k_window_attn_bwd(a, stream=stream)
        S.sif_k_rope(rope, bwd, stream=stream)
    step()
    torch.cuda.synchronize()
    pos, up = torch.arange(n), lambda x: x.cpu().double()
    for got, x, hh, back in ((tq, q, heads, False), (tk, k, h, False), (gq, dq, heads, True), (gk, dk, h, True)):
        val, off = turned(up(x).view(n, hh, d), pos, f, False, back=back)
        assert torch.all((up(got).view(n, hh, d) - val).abs() <= HALF * val.abs() + (1 + HALF) * off + 1e-30)
    val, tol = heads_attention(up(tq), up(tk), up(v), heads, h, d, visible(n, n, 0, 0), 0.125, up(do))
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert_within(got, val[name], tol[name], name)
    want = [x.clone() for x in (o, gq, gk, dv)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for _ in range(3):
        for x in (tq, tk, o, dq, dk, dv, gq, gk):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((o, gq, gk, dv), want))
