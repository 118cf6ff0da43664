"""The choice of a token on the GPU against its definition: every limit alone and together, ties, rows with nothing, numbers at their ends."""
import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from rows_reference import sample

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV


def _run(logits, vocab, u, pad=0, **kw):
    """logits [n][vocab] on the host, u [n]; settings as numbers or lists.  Returns tokens, log probabilities and how many were left."""
    n = logits.shape[0]
    ld = -(-vocab // 8) * 8 + pad
    wide = torch.full((n, ld), 1e30, dtype=logits.dtype, device=DEV)      # (what stands behind a row must not be chosen)
    wide[:, :vocab] = logits.to(DEV)
    token, kept, logprob = torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.full((n,), 7.0, device=DEV)
    given = {k: torch.tensor(x, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) if isinstance(x, list) else x for k, x in kw.items()}
    S.sif_k_sample(S.sample_args(wide, token, n, vocab, random=torch.tensor(u, dtype=torch.float32, device=DEV), logprob=logprob, kept=kept, **given))
    torch.cuda.synchronize()
    return token.cpu().tolist(), logprob.cpu().tolist(), kept.cpu().tolist()


def _check(logits, u, pad=0, **kw):
    vocab = logits.shape[1]
    got = _run(logits, vocab, u, pad, **kw)
    x = logits.double().numpy()
    at = lambda v, i: float(np.float32(v[i] if isinstance(v, list) else v)) if not isinstance(v, int) else v      # noqa: E731
    for i in range(len(u)):
        settings = {k: (v[i] if isinstance(v, list) else v) if k == "top_k" else at(v, i) for k, v in kw.items()}
        token, logprob, kept = sample(x[i], float(np.float32(u[i])), **settings)
        assert (got[0][i], got[2][i]) == (token, kept), (i, settings, u[i], got[0][i], token, got[2][i], kept)
        # a log probability is rounded to fp32 once
        assert got[1][i] == logprob if math.isinf(logprob) else abs(got[1][i] - logprob) <= 2.0 ** -24 * abs(logprob) + 1e-9, (i, got[1][i], logprob)


def _logits(seed, n, vocab, dtype, spread=3.0):
    return (spread * torch.randn(n, vocab, generator=torch.Generator().manual_seed(seed))).to(dtype)


LIMITS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=20, top_p=0.8), dict(top_p=0.95, min_p=0.02), dict(top_k=50, min_p=0.1),
          dict(temperature=1.4, top_k=100, top_p=0.9, min_p=0.01), dict(temperature=0.0), dict(temperature=0.0, top_k=3, top_p=0.5)]


@pytest.mark.parametrize("limits", LIMITS, ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 7, 8, 300, 4099])
def test_limits(vocab, dtype, limits):
    rng = random.Random(vocab)
    n = 24
    _check(_logits(vocab, n, vocab, dtype), [rng.random() for _ in range(n)], pad=rng.choice((0, 8, 40)), **limits)


@pytest.mark.parametrize("vocab,dtype", [(50257, torch.bfloat16), (50304, torch.float32), (65536, torch.float32), (65537, torch.float32), (131072, torch.bfloat16), (131080, torch.bfloat16), (262144, torch.float32),
                                         (262144, torch.bfloat16)], ids=str)
def test_large_vocabularies(vocab, dtype):
    rng = random.Random(vocab)
    n = len(LIMITS)
    logits, u = _logits(3, n, vocab, dtype, 2.0), [rng.random() for _ in range(n)]
    get = lambda name, off: [x.get(name, off) for x in LIMITS]      # noqa: E731
    _check(logits, u, temperature=get("temperature", 1.0), top_k=get("top_k", 0), top_p=get("top_p", 1.0), min_p=get("min_p", 0.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_equal_logits(dtype):
    """All equal, and a few values many times: counts and shares are exact, the lowest numbers win."""
    n, vocab = 20, 1000
    u = [i / n for i in range(n)]
    _check(torch.zeros(n, vocab, dtype=dtype), u, top_k=[1, 2, 10, 500, 999, 1000, 1001, 0] + [7] * 12)
    _check(torch.zeros(n, vocab, dtype=dtype), u, top_p=[0.5, 0.25, 0.001, 0.0, -1.0, 0.125, 0.75, 0.999] + [0.3] * 12)
    few = torch.randint(0, 4, (n, vocab), generator=torch.Generator().manual_seed(5)).to(dtype)
    _check(few, u, top_k=[300] * 10 + [100] * 10, top_p=[0.5 + 0.02 * i for i in range(n)])
    _check(few * 10, u, top_p=0.6)
    _check(few, u, min_p=[0.3, 0.4, 0.1, 1.0, 2.0] * 4)
    zeros = torch.zeros(n, vocab, dtype=dtype)
    zeros[:, ::2] = -0.0                                   # the same number
    _check(zeros, u, top_k=3)
    _check(zeros, u, temperature=0.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_without_tokens_and_tokens_that_are_none(dtype):
    x = _logits(6, 8, 500, dtype)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, :499] = -math.inf
    x[3, 100:] = math.nan
    x[4, 7], x[4, 400] = math.inf, math.inf
    x[5, 1::2] = -math.inf
    x[6] = torch.where(torch.arange(500) == 250, x[6], torch.tensor(-math.inf, dtype=dtype))
    x[7, 0] = math.nan
    u = [0.3, 0.5, 0.99, 0.7, 0.6, 0.999, 0.0, 0.4]
    for kw in (dict(), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=400, top_p=0.5, min_p=0.01)):
        _check(x, u, **kw)


def test_numbers_at_their_ends():
    x = _logits(7, 12, 777, torch.float32)
    u = [0.0, -1.0, math.nan, 1.0, 2.0, math.inf, 1 - 2.0 ** -24, 2.0 ** -24, 1e-30, -math.inf, 0.5, 0.25]
    for kw in (dict(), dict(top_k=5), dict(top_p=0.5)):
        _check(x, u, **kw)
    _check(x, [0.5] * 12, top_k=[-5, 0, 1, 776, 777, 778, 2 ** 31 - 1, -2 ** 31, 2, 3, 4, 5])
    _check(x, [0.9] * 12, top_p=[0.0, -1.0, 1.0, 2.0, math.inf, -math.inf, 1e-30, 1 - 2.0 ** -24, 0.5, 1e-3, 0.1, 0.01])
    _check(x, [0.9] * 12, min_p=[0.0, -1.0, 1.0, 2.0, math.inf, -math.inf, 1e-30, 0.5, 0.1, 1e-3, 0.999, 0.2])
    _check(x, [0.9] * 12, temperature=[0.0, -1.0, math.nan, 1e-30, 1e-40, 0.01, 100.0, 1e30, 3e38, 1.0, 1e-3, 10.0])
    _check(x * 1e37, [0.4] * 12, temperature=[1.0, 1e37, 1e38, 3e38] * 3)
    off = _run(x, 777, [0.5] * 12, top_p=[math.nan] * 12, min_p=[math.nan] * 12)
    assert off == _run(x, 777, [0.5] * 12)
    hot = _run(x, 777, [0.5] * 12, temperature=[math.inf] * 12)
    assert hot[0] == [388] * 12 and hot[2] == [777] * 12
    assert _run(x, 777, [0.5] * 12, temperature=[math.inf] * 12, min_p=1.0)[0] == [388] * 12
    y = torch.zeros(4, 777)
    y[:, ::3], y[:, 1::3] = -80.0, -43.0                   # probabilities of 2^-115 and 2^-62
    _check(y, [0.1, 0.4, 0.7, 0.99], min_p=[1e-34, 1e-36, 1e-18, 1e-19])
    _check(y, [0.1, 0.4, 0.7, 0.99], min_p=[1e-34, 1e-36, 1e-18, 1e-19], top_k=500)
    _check(y, [0.1, 0.4, 0.7, 0.99], min_p=[1e-34, 1e-36, 1e-18, 1e-19], top_k=600, top_p=0.9)


def test_tokens_follow_the_random_number():
    """Over a grid of random numbers: tokens never decrease, and each gets its share."""
    vocab, n = 50, 4096
    x = _logits(8, 1, vocab, torch.float32, 1.5)
    got = _run(x.expand(n, -1).contiguous(), vocab, [i / n for i in range(n)], temperature=0.9)[0]
    assert got == sorted(got)
    p = torch.softmax(x[0].double() / 0.9, 0)
    count = torch.bincount(torch.tensor(got), minlength=vocab)
    assert torch.all((count - n * p).abs() <= 1.0 + 1e-6)


def test_only_a_token_is_asked_for():
    x, u = _logits(9, 3, 1000, torch.bfloat16).to(DEV), torch.tensor([0.1, 0.5, 0.9], device=DEV)
    a, b = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    S.sif_k_sample(S.sample_args(x, a, 3, 1000, random=u, top_k=10))
    S.sif_k_sample(S.sample_args(x, b, 3, 1000, random=u, top_k=10, kept=torch.zeros(3, dtype=torch.int32, device=DEV), logprob=torch.zeros(3, device=DEV)))
    assert torch.equal(a, b)
    S.sif_k_sample(S.sample_args(x, a, 3, 1000, temperature=0.0))
    assert a.cpu().tolist() == x.float().argmax(1).cpu().tolist()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_tokens_far_below_the_largest(dtype):
    """Some tokens far above the others, whose probabilities are nothing beside theirs: they count among what is left all the same."""
    for vocab in (900, 20000):
        x = _logits(10, 8, vocab, dtype, 1.0)
        x[:, 123], x[4:, 7] = 1000.0, 900.0
        u = [0.0, 0.3, 0.6, 0.99] * 2
        for kw in (dict(top_k=50), dict(top_k=3), dict(top_k=600), dict(top_k=50, min_p=1e-30), dict(top_k=50, top_p=0.9), dict(temperature=30.0, top_k=40), dict(temperature=400.0, top_k=300, top_p=0.8), dict(top_p=0.5)):
            _check(x, u, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5003, 70000])
def test_many_equal_logits(vocab, dtype):
    """More equal ones than a list holds, on both sides of the border and in all parts of the row."""
    n = 12
    u = [(i + 0.5) / n for i in range(n)]
    zeros = torch.zeros(n, vocab, dtype=dtype)
    _check(zeros, u, top_k=[1, 63, 512, 513, 1024, 1025, 3000, vocab - 1, vocab, 2049, 4096, 0])
    _check(zeros, u, top_p=[0.5, 0.001, 0.999, 0.25, 1e-6, 0.75, 0.1, 0.9, 0.3, 0.6, 0.05, 0.8])
    few = torch.randint(0, 4, (n, vocab), generator=torch.Generator().manual_seed(12)).to(dtype)
    few[6:, vocab // 3:] = few[6:, vocab // 3:].clamp(max=1)      # the most probable ones at the row's start
    _check(few, u, top_k=[vocab // 3 + 17 * i for i in range(n)])
    _check(few, u, top_p=[0.4 + 0.05 * i for i in range(n)])
    _check(few, u, top_k=vocab // 2, top_p=[0.3 + 0.05 * i for i in range(n)], min_p=[0.0, 0.04, 0.05, 0.1, 0.13, 0.14, 0.3, 0.36, 0.37, 0.5, 1.0, 0.01])
    _check(few, u, top_k=2000, min_p=0.2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("descending", [False, True])
def test_rows_in_order(descending, dtype):
    """All that is left lies in one part of the row."""
    n, vocab = 10, 60001
    x = _logits(13, n, vocab, dtype, 2.0).sort(1, descending=descending)[0]
    u = [(i + 0.5) / n for i in range(n)]
    for kw in (dict(top_k=[1, 30, 100, 255, 257, 500, 512, 513, 900, 1100]), dict(top_p=0.02), dict(top_p=0.9), dict(top_p=0.6, temperature=0.5), dict(min_p=0.05), dict(top_k=30000, top_p=0.7, min_p=0.001), dict()):
        _check(x, u, **kw)


def test_logits_large_and_small_over_long_rows():
    """Steps of the logit far finer and far coarser than the numbers."""
    n, vocab = 9, 6007
    x = _logits(14, n, vocab, torch.float32, 2.0)
    u = [(i + 0.37) / n for i in range(n)]
    t = [1e-3, 0.03, 1.0, 1e2, 1e5, 1e9, 1e-8, 1e30, 0.3]
    for scale in (1e-30, 1e-4, 1.0, 1e4):
        for kw in (dict(top_p=0.5), dict(top_k=600), dict(top_k=40), dict(top_k=3000, top_p=0.7), dict(min_p=0.3)):
            _check(x * scale, u, temperature=t, **kw)


def test_rows_at_once_on_streams_and_in_a_graph():
    """Two calls under way at the same time, and a captured one whose numbers change between replays."""
    n, vocab = 40, 20000
    x, y = _logits(15, n, vocab, torch.bfloat16).to(DEV), _logits(16, n, vocab, torch.float32).to(DEV)
    u = torch.rand(n, generator=torch.Generator().manual_seed(17)).to(DEV)
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for _ in range(4)]
    S.sif_k_sample(S.sample_args(x, out[0], n, vocab, random=u, top_p=0.9))
    S.sif_k_sample(S.sample_args(y, out[1], n, vocab, random=u, top_k=300))
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        out[2].zero_(), out[3].zero_()
        torch.cuda.synchronize()
        S.sif_k_sample(S.sample_args(x, out[2], n, vocab, random=u, top_p=0.9), stream=one)
        S.sif_k_sample(S.sample_args(y, out[3], n, vocab, random=u, top_k=300), stream=two)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    graph, v = torch.cuda.CUDAGraph(), u.clone()
    with torch.cuda.graph(graph):
        S.sif_k_sample(S.sample_args(x, out[2], n, vocab, random=v, top_p=0.9), stream=torch.cuda.current_stream())
    for turn in range(4):
        v.copy_((u + 0.21 * turn) % 1.0)
        graph.replay()
        S.sif_k_sample(S.sample_args(x, out[0], n, vocab, random=v, top_p=0.9))
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2])


def test_rows_past_32_bits():
    n, vocab = 16700, 131072                               # 4.4 GB
    x = torch.zeros(n, vocab, dtype=torch.bfloat16, device=DEV)
    hot = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(1))
    x[torch.arange(n, device=DEV), hot.to(DEV)] = 30.0
    token = torch.zeros(n, dtype=torch.int32, device=DEV)
    S.sif_k_sample(S.sample_args(x, token, n, vocab, random=torch.full((n,), 0.5, device=DEV), top_k=4))
    assert token.cpu().tolist() == hot.tolist()
