"""Rotary positions, writing into a paged cache with the rotation on the way and reading back, attention over a cache held in 4 bits, and
the choice of a token from logits, as cases that can be timed and compared.

Four kinds of pass, as a program on this library makes them (`own`), and the same in elementary torch operations:

  rope     queries and keys are turned by their positions: forward, or forward and the gradients back through it
  append   new tokens' queries and keys are turned, keys and values written to a paged cache in bf16, 8 or 4 bits; where the cache is not
           held in bf16 all its tokens' keys and values are then read back as rows, as the attention of a prompt's next piece takes them
  decode   attention of one new token per sequence over a paged cache in 4 bits
  sample   one token per row of logits: temperature, the k most probable, the most probable that hold p together, those of at least a
           fraction of the most probable one; random numbers are inputs

Layouts: rows of q, k and v are tokens, a head is a column slice.  A cache in bf16 or e4m3 holds keys as [layer][page][kv head][token][d] and
values as [layer][page][kv head][d][token].  In 4 bits (e2m1: sign, two bits of exponent, one of mantissa) 32 consecutive d of a token share a
power of two, one byte b for 2^(b - 127), 255 for NaN; a page of a kv head holds, in this order,

  keys     [token][d / 2] bytes, the lower half of byte i is d = 2 i, the upper one 2 i + 1;   [d / 32][token] powers
  values   [d / 32][16][token] bytes, the lower half of byte (b, c) is d = 32 b + c, the upper one d + 16;   [token][d / 32] powers

Head counts and sizes are those of the configurations in synth_inputs.py, perf/cases.py and perf/operators.py, or generic ones.
"""
import math

import torch

own = False

DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn


# ---- cases -------------------------------------------------------------------------------------------------------
def _turn(**kw):
    """Which elements are turned how: `rot` of a head's d, in halves or neighbours, frequencies base^(-2 i / rot) and how they are scaled."""
    return dict(dict(layout="half", base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, trained=4096, magnitude=1.0), **kw)


def _rope(**kw):
    return dict(dict(kind="rope", train=False, listed_positions=False, first=0), **_turn(**kw))


def _append(**kw):
    return dict(dict(kind="append", layers=1, new_min=1, new_max=1), **_turn(**kw))


def _decode(**kw):
    return dict(dict(kind="decode", window=0, sinks=0), **kw)


def _sample(**kw):
    return dict(dict(kind="sample", mixed=False, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, banned=0.0), **kw)


def listed():
    return [
        # one request of odd length at an idle instance: latency
        _rope(name="rope_small", batch=1, seq=77, heads=12, kv_heads=12, d_head=64, rot=64, layout="interleaved"),
        # the decoder's training step, one layer: queries and keys forward, their gradients back
        _rope(name="rope_train", train=True, batch=8, seq=1024, heads=12, kv_heads=12, d_head=64, rot=64),
        # documents at positions far beyond the trained length, half of each head turned, frequencies scaled by parts
        _rope(name="rope_far", batch=2, seq=16381, heads=32, kv_heads=8, d_head=128, rot=64, scaling="parts", factor=32.0, magnitude=1.35, listed_positions=True),
        # four sequences, one new token each: latency
        _append(name="append_small", dtype="bf16", n=4, len_min=5, len_max=300, heads=12, kv_heads=12, d_head=64, rot=64, page=16),
        # a full batch, one new token each
        _append(name="append_step", dtype="bf16", n=128, len_min=1, len_max=800, heads=32, kv_heads=8, d_head=128, rot=128, page=16, scaling="linear", factor=4.0),
        # prompts of 1 to 611 tokens into a cache of 8 bits, half of each head turned in neighbours
        _append(name="append_prompts_8bit", dtype="e4m3", n=9, len_min=0, len_max=40, new_min=1, new_max=611, heads=12, kv_heads=4, d_head=64, rot=32, page=16, layout="interleaved"),
        # pieces of long prompts behind what a cache of 4 bits already holds
        _append(name="append_prompts_4bit", dtype="e2m1", n=24, len_min=0, len_max=700, new_min=3, new_max=2047, heads=32, kv_heads=8, d_head=128, rot=128, page=64, scaling="base", factor=8.0),
        # one request of odd length at an idle instance: latency
        _decode(name="decode_small_4bit", n=1, len_min=77, len_max=77, heads=12, kv_heads=12, d_head=64, page=16),
        # a full batch of requests of very different lengths
        _decode(name="decode_batch_4bit", n=64, len_min=1, len_max=8192, heads=32, kv_heads=8, d_head=128, page=16),
        # one very long context
        _decode(name="decode_long_4bit", n=1, len_min=262011, len_max=262011, heads=32, kv_heads=8, d_head=128, page=64),
        # one request's next token
        _sample(name="sample_one", dtype="bf16", n=1, vocab=50257, temperature=0.8, top_k=50, top_p=0.95),
        # a batch of requests, each with settings of its own: greedy, every single filter, all of them, none
        _sample(name="sample_batch", dtype="f32", n=256, vocab=50304, mixed=True, banned=0.01),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    kv = rng.choice([h for h in (1, 2, 4, 8, 12, 16) if h <= most])
    return dict(heads=kv * rng.choice([g for g in (1, 2, 3, 4, 8) if kv * g <= most]), kv_heads=kv)


def _scaled(rng):
    how = rng.choice(("plain", "linear", "base", "parts"))
    return dict(layout=rng.choice(("half", "interleaved")), base=rng.choice((10000.0, 500000.0)), scaling=how, factor=1.0 if how == "plain" else rng.uniform(1.5, 40.0),
                trained=rng.choice((1024, 4096, 8192)), magnitude=1.0 if rng.random() < 0.7 else rng.uniform(1.0, 1.5))


def _draw(rng):
    pick = rng.random()
    if pick < 0.25:
        d = rng.choice((32, 64, 64, 80, 128, 128, 256))
        return _rope(train=rng.random() < 0.5, batch=rng.randint(1, 8), seq=_log(rng, 1, 17000), d_head=d, rot=16 * rng.randint(1, d // 16), first=rng.choice((0, 0, rng.randint(1, 200000))),
                     listed_positions=rng.random() < 0.4, **_heads(rng, 32), **_scaled(rng))
    if pick < 0.55:
        d = rng.choice((64, 128))
        lo, new = rng.randint(0, 50), rng.choice((1, 1, _log(rng, 2, 3000)))
        return _append(dtype=rng.choice(("bf16", "e4m3", "e2m1", "e2m1")), n=_log(rng, 1, 128), len_min=lo, len_max=lo + _log(rng, 1, 1000), new_min=1 if new == 1 else rng.randint(0, new), new_max=new,
                       d_head=d, rot=16 * rng.randint(1, d // 16), page=rng.choice((16, 32, 64, 128)), layers=rng.randint(1, 3), **_heads(rng, 32), **_scaled(rng))
    if pick < 0.75:
        lo, window = _log(rng, 1, 4000), rng.choice((0, 0, _log(rng, 16, 4096)))
        return _decode(n=_log(rng, 1, 128), len_min=lo, len_max=lo + _log(rng, 1, 60000), page=rng.choice((16, 32, 64, 128)), d_head=rng.choice((64, 128)), window=window,
                       sinks=rng.choice((0, 4, 33)) if window else 0, **_heads(rng, 48))
    return _sample(dtype=rng.choice(("bf16", "f32")), n=_log(rng, 1, 400), vocab=_log(rng, 200, 140000), mixed=rng.random() < 0.4, temperature=rng.choice((1.0, rng.uniform(0.2, 1.6))),
                   top_k=rng.choice((0, 0, _log(rng, 1, 2000))), top_p=rng.choice((1.0, rng.uniform(0.3, 0.99))), min_p=rng.choice((0.0, rng.uniform(0.01, 0.2))), banned=rng.choice((0.0, 0.02)))


def draw(rng):
    listings = listed()
    while True:
        c = _draw(rng)
        most = max((work(x) for x in listings if x["kind"] == c["kind"]), key=lambda w: w["bytes"])
        if work(c)["bytes"] <= most["bytes"] and _held(c) <= 4e9:
            return c


# ---- shapes, and the work a pass cannot do without ----------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths over a range, in no order."""
    if n == 1:
        return [hi]
    got = [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return [got[i * 7 % n] for i in range(n)] if n % 7 else got[::-1]


def _old(c):
    return _spread(c["n"], c["len_min"], c["len_max"])


def _new(c):
    """New tokens of each sequence of an append case, the longest prompts not behind the longest contexts; at least one in all."""
    return [max(m, 1) if i == 0 else m for i, m in enumerate(_spread(c["n"], c["new_min"], c["new_max"])[::-1])]


def _lengths(c):
    return [a + b for a, b in zip(_old(c), _new(c))] if c["kind"] == "append" else _old(c)


BYTES = {"bf16": 2.0, "e4m3": 1.0, "e2m1": 17.0 / 32.0}


def _held(c):
    """Bytes of the plain form's largest tensor."""
    if c["kind"] == "decode":
        return 4.0 * c["n"] * c["len_max"] * c["kv_heads"] * c["d_head"]
    if c["kind"] == "append":
        return 8.0 * sum(_lengths(c)) * max(c["heads"], c["kv_heads"]) * c["d_head"]
    return 8.0 * c["n"] * c["vocab"] if c["kind"] == "sample" else 4.0 * c["batch"] * c["seq"] * c["heads"] * c["d_head"]


def _pairs(sq, sk, window, sinks):
    total = 0
    for p in range(sk - sq, sk):
        near = min(p + 1, window) if window else p + 1
        total += near + min(sinks, p + 1 - near)
    return total


def work(c):
    """Every input and output once; of a rotation the multiplications and additions, of attention its two products over visible keys."""
    if c["kind"] == "rope":
        rows, h = c["batch"] * c["seq"], c["heads"] + c["kv_heads"]
        times = 2 if c["train"] else 1
        return {"bytes": times * 4.0 * rows * h * c["d_head"] + (4.0 * rows if c["listed_positions"] else 0.0), "flops": times * 3.0 * rows * h * c["rot"]}
    if c["kind"] == "append":
        rows, width = sum(_new(c)), c["kv_heads"] * c["d_head"]
        total = 4.0 * rows * c["heads"] * c["d_head"] + 2.0 * rows * width * (2.0 + BYTES[c["dtype"]])
        if c["dtype"] != "bf16":
            total += 2.0 * sum(_lengths(c)) * width * (2.0 + BYTES[c["dtype"]])
        return {"bytes": total, "flops": 3.0 * rows * (c["heads"] + c["kv_heads"]) * c["rot"]}
    if c["kind"] == "decode":
        seen = sum(_pairs(1, m, c["window"], c["sinks"]) for m in _lengths(c))
        return {"bytes": 2.0 * BYTES["e2m1"] * seen * c["kv_heads"] * c["d_head"] + 4.0 * c["n"] * c["heads"] * c["d_head"], "flops": 4.0 * seen * c["heads"] * c["d_head"]}
    return {"bytes": (2.0 if c["dtype"] == "bf16" else 4.0) * c["n"] * c["vocab"] + 12.0 * c["n"], "flops": 2.0 * c["n"] * c["vocab"]}


# ---- numbers in 4 bits -------------------------------------------------------------------------------------------
def _lut():
    """The values of a byte's lower and upper half."""
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEV)
    i = torch.arange(256, device=DEV)
    return torch.stack([e2m1[i & 15], e2m1[i >> 4]], 1)


def _codes(x):
    """x [..., d] as e2m1 codes (0 .. 15) and the powers' bytes [..., d / 32]: the smallest power by which no element exceeds 7, each
    element to the nearest value, in the middle to the even one."""
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(torch.nan_to_num(top, 0.0, 3.0e38))
    e = torch.where(m <= 0.875, e - 3, e - 2)
    e = torch.where(top == 0, -127, e).clamp(-127, 127)
    z = torch.ldexp(y, -e).abs()
    code = (z > 0.25).to(torch.uint8) + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5.0)
    code = code | (torch.signbit(y).to(torch.uint8) << 3)
    byte = torch.where(top.isnan(), 255, e + 127).to(torch.uint8)
    return torch.where(top.isnan(), 0, code).flatten(-2), byte.squeeze(-1)


def _pow(byte):
    return torch.where(byte == 255, math.nan, torch.exp2(byte.float() - 127.0))


def _parts(c, pool, of_values):
    """A page's bytes and powers as views, by token: [page][kv head][token][d / 2] and [page][kv head][token][d / 32]."""
    d, page = c["d_head"], c["page"]
    data, power = pool[..., :page * d // 2], pool[..., page * d // 2:]
    if of_values:
        return data.unflatten(-1, (d // 2, page)).transpose(-1, -2), power.unflatten(-1, (page, d // 32))
    return data.unflatten(-1, (page, d // 2)), power.unflatten(-1, (d // 32, page)).transpose(-1, -2)


def _packed(code, of_values):
    if of_values:
        y = code.unflatten(-1, (-1, 2, 16))
        return (y[..., 0, :] | (y[..., 1, :] << 4)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpacked(data, power, of_values):
    """Bytes [..., d / 2] and powers [..., d / 32] as values [..., d]."""
    y = _lut()[data.long()]                              # [..., d / 2, 2]
    y = y.unflatten(-2, (-1, 16)).transpose(-1, -2).flatten(-3) if of_values else y.flatten(-2)
    return (y.unflatten(-1, (-1, 32)) * _pow(power)[..., None]).flatten(-2)


# ---- states ------------------------------------------------------------------------------------------------------
def _bf16(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _pools(gen, c, layers, n_pages):
    """Keys and values of a cache."""
    h, d, page = c["kv_heads"], c["d_head"], c["page"]
    dtype = c.get("dtype", "e2m1")
    if dtype == "e2m1":
        s = {}
        for name in ("k", "v"):
            pool = torch.empty(layers, n_pages, h, page * d * 17 // 32, device=DEV, dtype=torch.uint8)
            data, power = _parts(c, pool, name == "v")
            step = max(1, (1 << 25) // (h * page * d))
            for i in range(layers):
                for a in range(0, n_pages, step):
                    code, byte = _codes(torch.randn(min(step, n_pages - a), h, page, d, generator=gen, device=DEV))
                    data[i, a:a + step], power[i, a:a + step] = _packed(code, name == "v"), byte
            s[name] = pool
        return s | dict(k_scale=None, v_scale=None)

    def some(*shape):
        x = torch.empty(shape, device=DEV, dtype=torch.bfloat16 if dtype == "bf16" else E4M3)
        for part in x.view(-1).split(1 << 27):
            y = torch.randn(part.numel(), generator=gen, device=DEV, dtype=torch.float32)
            part.copy_(y if dtype == "bf16" else (y * 64.0).clamp(-448.0, 448.0))
        return x
    scale = lambda: (0.8 + 0.4 * torch.rand(layers, h, generator=gen, device=DEV)) / 64.0 if dtype == "e4m3" else None      # noqa: E731
    return dict(k=some(layers, n_pages, h, page, d), v=some(layers, n_pages, h, d, page), k_scale=scale(), v_scale=scale())


def _tables(gen, c, lens):
    """Sequences in some of a few more slots than there are, on pages of a shuffled pool."""
    page, n = c["page"], len(lens)
    count = torch.tensor([-(-m // page) for m in lens], device=DEV)
    width, n_pages = max(1, int(count.max())), int(count.sum()) + 3
    slot = torch.arange(width, device=DEV)[None, :].expand(n, width)
    order = torch.randperm(n_pages, generator=gen, device=DEV)
    rows = torch.where(slot < count[:, None], order[((count.cumsum(0) - count)[:, None] + slot).clamp(max=n_pages - 1)], -1).to(torch.int32)
    seqs = torch.randperm(n + 2, generator=gen, device=DEV)[:n]
    table, lengths, refs = torch.full((n + 2, width), -1, device=DEV, dtype=torch.int32), torch.zeros(n + 2, device=DEV, dtype=torch.int32), torch.zeros(n_pages, device=DEV, dtype=torch.int32)
    table[seqs], lengths[seqs] = rows, torch.tensor(lens, device=DEV, dtype=torch.int32)
    refs[order[:int(count.sum())]] = 1
    return dict(table=table, lengths=lengths, refs=refs, seqs=seqs.to(torch.int32)), n_pages


def _starts(lens):
    return torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "rope":
        rows, wq, wk = c["batch"] * c["seq"], c["heads"] * c["d_head"], c["kv_heads"] * c["d_head"]
        s |= dict(q=_bf16(gen, rows, wq), k=_bf16(gen, rows, wk))
        if c["train"]:
            s |= dict(dq=_bf16(gen, rows, wq), dk=_bf16(gen, rows, wk))
        if c["listed_positions"]:
            s["positions"] = (torch.arange(rows, device=DEV) % c["seq"] + torch.randint(0, 200000, (c["batch"], 1), generator=gen, device=DEV).expand(-1, c["seq"]).reshape(-1)).to(torch.int32)
        return s | {"to_" + x: torch.empty_like(s[x]) for x in ("q", "k", "dq", "dk") if x in s}
    if c["kind"] == "sample":
        ld = -(-c["vocab"] // 8) * 8
        x = 2.0 * torch.randn(c["n"], ld, generator=gen, device=DEV)
        # a few tokens that the text makes likely
        likely = torch.rand(c["n"], ld, generator=gen, device=DEV) < 40.0 / c["vocab"]
        x = torch.where(likely, 4.0 + 3.0 * torch.randn(c["n"], ld, generator=gen, device=DEV), x)
        if c["banned"]:
            x.masked_fill_(torch.rand(c["n"], ld, generator=gen, device=DEV) < c["banned"], -math.inf)
        s["logits"] = x if c["dtype"] == "f32" else x.to(torch.bfloat16)
        s["random"] = torch.rand(c["n"], generator=gen, device=DEV)
        if c["mixed"]:
            which = torch.arange(c["n"], device=DEV) % 8
            r = lambda lo, hi: lo + (hi - lo) * torch.rand(c["n"], generator=gen, device=DEV)      # noqa: E731
            s["temperature"] = torch.where(which == 0, 0.0, r(0.4, 1.5))
            s["top_k"] = torch.where((which == 1) | (which >= 6), r(1.0, 200.0).to(torch.int32), 0).to(torch.int32)
            s["top_p"] = torch.where((which == 2) | (which >= 5), r(0.5, 0.99), 1.0)
            s["min_p"] = torch.where((which == 3) | (which == 7), r(0.01, 0.2), 0.0)
        return s | dict(token=torch.zeros(c["n"], device=DEV, dtype=torch.int32), kept=torch.zeros(c["n"], device=DEV, dtype=torch.int32), logprob=torch.zeros(c["n"], device=DEV))
    book, n_pages = _tables(gen, c, _lengths(c))
    s |= book | _pools(gen, c, c.get("layers", 1), n_pages)
    if c["kind"] == "decode":
        s["q"] = _bf16(gen, c["n"], c["heads"] * c["d_head"])
        return s | dict(o=torch.empty_like(s["q"]), lse=torch.empty(c["n"], c["heads"], device=DEV))
    rows, wk = sum(_new(c)), c["kv_heads"] * c["d_head"]
    s |= dict(q=_bf16(gen, rows, c["heads"] * c["d_head"]), k_new=_bf16(gen, rows, wk), v_new=_bf16(gen, rows, wk), starts=_starts(_new(c)))
    s["to_q"] = torch.empty_like(s["q"])
    if c["dtype"] != "bf16":
        s["all"] = _starts(_lengths(c))
        s |= {x: torch.empty(sum(_lengths(c)), wk, device=DEV, dtype=torch.bfloat16) for x in ("k_rows", "v_rows")}
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _frequencies(c):
    """Angle per token of each pair, in 64 bits."""
    i = torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"]
    base, factor = c["base"], c["factor"]
    if c["scaling"] == "base":
        base *= factor ** (c["rot"] / (c["rot"] - 2))
    f = base ** -i
    if c["scaling"] == "linear":
        return f / factor
    if c["scaling"] == "parts":
        keep = ((c["trained"] * f / (2 * math.pi) - c["low"]) / (c["high"] - c["low"])).clamp(0.0, 1.0)
        return keep * f + (1 - keep) * f / factor
    return f


def _turned(c, x, pos, heads, back=False, wide=torch.float32):
    """Rows of heads, each turned by its position; angles in 64 bits, the rest in `wide`."""
    angle = pos.double()[:, None] * _frequencies(c)
    m = c["magnitude"]
    cos, sin = (m * angle.cos()).to(wide)[:, None, :], (m * angle.sin()).to(wide)[:, None, :]
    if back:
        sin = -sin
    y = x.to(wide).view(x.shape[0], heads, c["d_head"]).clone()
    r = c["rot"]
    first, second = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y


def _positions(s):
    c = s["case"]
    return s["positions"] if "positions" in s else torch.arange(s["q"].shape[0], device=DEV) % c["seq"] + c["first"]


def _plain_rope(s):
    c = s["case"]
    pos, out = _positions(s), {}
    for x in ("q", "k", "dq", "dk"):
        if x in s:
            out[x] = _turned(c, s[x], pos, c["heads"] if "q" in x else c["kv_heads"], x[0] == "d").to(torch.bfloat16).view_as(s[x])
    return out


def _places(s, starts, count):
    """Page, place in it and position of the rows starts[i] .. starts[i + 1] - 1, the last tokens of sequence i of the list."""
    row = torch.arange(count, device=DEV)
    i = torch.searchsorted(starts, row.to(torch.int32), right=True) - 1
    seq = s["seqs"].long()[i]
    pos = s["lengths"].long()[seq] - starts.long()[i + 1] + row
    return s["table"].long()[seq, pos // s["case"]["page"]], pos % s["case"]["page"], pos


def _plain_append(s):
    c = s["case"]
    layer, h, d, dtype = c["layers"] - 1, c["kv_heads"], c["d_head"], c["dtype"]
    at, off, pos = _places(s, s["starts"], s["q"].shape[0])
    out = {"q": _turned(c, s["q"], pos, c["heads"]).to(torch.bfloat16).view_as(s["q"])}
    # (a value next to a border between two of 8 or 4 bits goes to one or the other by its last bits)
    k = _turned(c, s["k_new"], pos, h, wide=torch.float32 if dtype == "bf16" else torch.float64)
    v = s["v_new"].view(-1, h, d).to(k.dtype)
    if dtype == "e2m1":
        for name, x in (("k", k), ("v", v)):
            data, power = _parts(c, s[name][layer], name == "v")
            code, byte = _codes(x)
            data[at, :, off], power[at, :, off] = _packed(code, name == "v"), byte
    elif dtype == "e4m3":
        held = lambda x, scale: (x / scale[layer].double()[None, :, None]).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)      # noqa: E731
        s["k"][layer].view(torch.uint8)[at, :, off] = held(k, s["k_scale"])
        s["v"][layer].view(torch.uint8).transpose(-1, -2)[at, :, off] = held(v, s["v_scale"])
    else:
        s["k"][layer][at, :, off] = k.to(torch.bfloat16)
        s["v"][layer].transpose(-1, -2)[at, :, off] = v.to(torch.bfloat16)
        return out | {"k": s["k"], "v": s["v"]}
    at, off, _ = _places(s, s["all"], s["k_rows"].shape[0])
    for name in ("k", "v"):
        if dtype == "e2m1":
            data, power = _parts(c, s[name][layer], name == "v")
            x = _unpacked(data[at, :, off], power[at, :, off], name == "v")
        else:
            pool = s[name][layer].view(torch.uint8)
            x = (pool if name == "k" else pool.transpose(-1, -2))[at, :, off].view(E4M3).float() * s[name + "_scale"][layer][None, :, None]
        out[name] = x.to(torch.bfloat16).reshape(-1, h * d)
    return out


def _seen(qpos, kpos, window, sinks):
    near = (kpos > qpos - window) if window else torch.ones_like(kpos <= qpos)
    return (kpos <= qpos) & (near | (kpos < sinks))


def _plain_decode(s):
    c = s["case"]
    n, h, g, d = c["n"], c["heads"], c["kv_heads"], c["d_head"]
    page, seqs = s["table"].long()[s["seqs"].long()].clamp(min=0), s["seqs"].long()
    x = []
    for name in ("k", "v"):
        data, power = _parts(c, s[name][0], name == "v")
        y = torch.empty(n, g, page.shape[1] * c["page"], d, device=DEV)
        for i in range(n):                               # (one sequence at a time: the indices of all would be larger than the values)
            a, b = (z[page[i]].transpose(0, 1).flatten(1, 2) for z in (data, power))
            y[i] = _unpacked(a, b, name == "v")
        x.append(y)
    k, v = x
    last = s["lengths"].long()[seqs][:, None] - 1
    seen = _seen(last, torch.arange(k.shape[2], device=DEV)[None, :], c["window"], c["sinks"])[:, None, None, :]
    q = s["q"].float().view(n, g, h // g, d)
    score = torch.where(seen, torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    o = torch.matmul(p / torch.where(total > 0, total, 1.0), v)
    return {"o": o.reshape(n, h * d).to(torch.bfloat16), "lse": lse.reshape(n, h)}


def _settings(s):
    """Temperature, k, p and the least fraction of every row, as columns in 64 bits."""
    c = s["case"]
    return [s[x].double()[:, None] if x in s else torch.full((c["n"], 1), float(c[x]), device=DEV, dtype=torch.float32).double() for x in ("temperature", "top_k", "top_p", "min_p")]


def _plain_sample(s):
    c = s["case"]
    temperature, top_k, top_p, min_p = _settings(s)
    x = s["logits"][:, :c["vocab"]].float()
    x, order = torch.sort(torch.where(x.isnan(), -math.inf, x), dim=1, descending=True, stable=True)
    x = x.double()
    rank = torch.arange(c["vocab"], device=DEV)[None, :]
    some = x[:, :1] > -math.inf
    w = torch.exp((x - torch.where(some, x[:, :1], 0.0)) / torch.where(temperature > 0, temperature, 1.0))
    keep = (x > -math.inf) & ((rank < top_k) | (top_k <= 0)) & ((rank < 1) | (temperature > 0))
    so_far = (w * keep).cumsum(1)
    before = torch.cat([torch.zeros_like(w[:, :1]), so_far[:, :-1]], 1)
    keep &= (before < top_p * so_far[:, -1:]) | (top_p >= 1.0) | (rank < 1)
    keep &= (w >= min_p) | (rank < 1)
    # in the order of the vocabulary: the first token at which the sum exceeds the random share of the whole
    left = torch.zeros_like(w).scatter_(1, order, w * keep)
    upto = left.cumsum(1)
    whole = upto[:, -1:]
    token = (upto <= s["random"].double()[:, None] * whole).sum(1, keepdim=True).clamp(max=c["vocab"] - 1)
    logprob = torch.log(left.gather(1, token) / whole)
    none = ~some[:, 0]
    return {"token": torch.where(none, -1, token[:, 0]).to(torch.int32), "logprob": torch.where(none, -math.inf, logprob[:, 0]).float(), "kept": keep.sum(1).to(torch.int32)}


# ---- the library's calls -----------------------------------------------------------------------------------------
def _handles(s):
    """What a program sets up once for its buffers: the rotation's table, argument structures and workspaces."""
    import paper_2503_02550_amd as S
    c = s["case"]
    if c["kind"] == "sample":
        get = lambda x: s.get(x, c[x])      # noqa: E731
        return S, S.sample_args(s["logits"], s["token"], n=c["n"], vocab=c["vocab"], random=s["random"], temperature=get("temperature"), top_k=get("top_k"), top_p=get("top_p"),
                                min_p=get("min_p"), logprob=s["logprob"], kept=s["kept"])
    if c["kind"] in ("rope", "append"):
        rope = S.rope_plan(c["rot"], layout=S.SIF_ROPE_HALF if c["layout"] == "half" else S.SIF_ROPE_INTERLEAVED, base=c["base"],
                           scaling={"plain": S.SIF_ROPE_PLAIN, "linear": S.SIF_ROPE_LINEAR, "base": S.SIF_ROPE_BASE, "parts": S.SIF_ROPE_PARTS}[c["scaling"]],
                           factor=c["factor"], low_turns=c["low"], high_turns=c["high"], trained_tokens=c["trained"], magnitude=c["magnitude"])
    if c["kind"] == "rope":
        where = dict(positions=s.get("positions"), seq=c["seq"], first=c["first"])
        sizes = dict(rows=s["q"].shape[0], heads=c["heads"], kv_heads=c["kv_heads"], d_head=c["d_head"])
        calls = [S.rope_args(s["q"], s["to_q"], k=s["k"], k_out=s["to_k"], **sizes, **where)]
        if c["train"]:
            calls.append(S.rope_args(s["dq"], s["to_dq"], k=s["dk"], k_out=s["to_dk"], inverse=True, **sizes, **where))
        return S, rope, calls
    dtype = {"bf16": S.SIF_BF16, "e4m3": S.SIF_E4M3, "e2m1": S.SIF_E2M1}[c.get("dtype", "e2m1")]
    cache = S.kv_cache(s["k"], s["v"], s["table"], s["lengths"], s["refs"], dtype=dtype, page_tokens=c["page"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    if c["kind"] == "append":
        return S, cache, rope, S.kv_append_args(s["k_new"], s["v_new"], n=c["n"], rows=s["q"].shape[0], layer=c["layers"] - 1, seqs=s["seqs"], starts=s["starts"], q=s["q"], q_out=s["to_q"], heads=c["heads"])
    a = S.attn_decode_args(s["q"], s["o"], n=c["n"], heads=c["heads"], window=c["window"], sinks=c["sinks"], max_tokens=c["len_max"], seqs=s["seqs"], lse=s["lse"])
    n = S.sif_attn_decode_workspace_bytes(cache, a)
    s["workspace"] = torch.empty(n, device=DEV, dtype=torch.uint8)
    S.set_workspace(a, s["workspace"], n)
    return S, cache, a


def _own(s):
    c = s["case"]
    if "handles" not in s:
        s["handles"] = _handles(s)
    if c["kind"] == "sample":
        S, a = s["handles"]
        S.sif_k_sample(a)
        return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}
    if c["kind"] == "rope":
        S, rope, calls = s["handles"]
        for a in calls:
            S.sif_k_rope(rope, a)
        return {x: s["to_" + x] for x in ("q", "k", "dq", "dk") if x in s}
    if c["kind"] == "decode":
        S, cache, a = s["handles"]
        S.sif_k_attn_decode(cache, a)
        return {"o": s["o"], "lse": s["lse"]}
    S, cache, rope, a = s["handles"]
    S.sif_k_kv_append(cache, rope, a)
    if c["dtype"] == "bf16":
        return {"q": s["to_q"], "k": s["k"], "v": s["v"]}
    S.sif_k_kv_read(cache, c["layers"] - 1, s["k_rows"], s["v_rows"], s["seqs"], c["n"], starts=s["all"], rows=s["k_rows"].shape[0])
    return {"q": s["to_q"], "k": s["k_rows"], "v": s["v_rows"]}


def run(s):
    if own:
        return _own(s)
    return {"rope": _plain_rope, "append": _plain_append, "decode": _plain_decode, "sample": _plain_sample}[s["case"]["kind"]](s)


# ---- the same in 64 bits -----------------------------------------------------------------------------------------
def _exact_turn(c, x, pos, heads, sign=1.0):
    """Pairs as complex numbers, times m e^(i sign p f)."""
    r, d = c["rot"], c["d_head"]
    out = x.double().view(-1, heads, d).clone()
    f = []
    for i in range(r // 2):
        base = c["base"] * c["factor"] ** (r / (r - 2.0)) if c["scaling"] == "base" else c["base"]
        w = base ** (-2.0 * i / r)
        if c["scaling"] == "linear":
            w /= c["factor"]
        if c["scaling"] == "parts":
            turns = c["trained"] * w / (2.0 * math.pi)
            share = min(1.0, max(0.0, (turns - c["low"]) / (c["high"] - c["low"])))
            w = share * w + (1.0 - share) * w / c["factor"]
        f.append(w)
    by = torch.polar(torch.full((len(pos), r // 2), c["magnitude"], device=DEV, dtype=torch.float64), sign * torch.outer(pos.double(), torch.tensor(f, device=DEV, dtype=torch.float64)))[:, None, :]
    part = out[..., :r]
    z = torch.complex(part[..., :r // 2].contiguous(), part[..., r // 2:].contiguous()) if c["layout"] == "half" else torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous())
    z = z * by
    out[..., :r] = torch.cat([z.real, z.imag], -1) if c["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return out


def _exact_4bit(x):
    """The values that e2m1 with a power of two per 32 holds for x."""
    grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 6.0, 0.5, 1.5, 3.0], device=DEV, dtype=torch.float64)      # even ones first: of two that are as near they are found
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -127.0)
    near = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    for k in (-1.0, -2.0, -3.0):                         # the smallest power that is enough
        e = torch.where((top > 0) & (top <= 7.0 * torch.exp2(near + k)), near + k, e)
    z = y * torch.exp2(-e)
    best, off = torch.zeros_like(z), torch.full_like(z, math.inf)
    for g in grid:
        d = (z.abs() - g).abs()
        best, off = torch.where(d < off, g, best), torch.minimum(d, off)
    return (torch.copysign(best, z) * torch.exp2(e)).flatten(-2)


def _exact_append(c, s):
    h, d, page, layer, dtype = c["kv_heads"], c["d_head"], c["page"], c["layers"] - 1, c["dtype"]
    lens, new, seqs, starts = _lengths(c), _new(c), s["seqs"].cpu().tolist(), s["starts"].cpu().tolist()
    pos = torch.cat([torch.arange(m - n, m, device=DEV) for m, n in zip(lens, new)])
    fresh = {"k": _exact_turn(c, s["k_new"], pos, h), "v": s["v_new"].double().view(-1, h, d)}
    out = {"q": _exact_turn(c, s["q"], pos, c["heads"]).view(-1, c["heads"] * d)}
    for name in ("k", "v"):
        rows = []
        x = fresh[name]
        pool = s[name].clone() if dtype == "bf16" else None
        if dtype == "e2m1":
            x = _exact_4bit(x)
        if dtype == "e4m3":
            scale = s[name + "_scale"][layer].double()[None, :, None]
            x = (x / scale).clamp(-448.0, 448.0).to(E4M3).double() * scale
        for i, (m, n, q) in enumerate(zip(lens, new, seqs)):
            at = torch.arange(m - n, m, device=DEV)
            mine = x[starts[i]:starts[i + 1]]
            pages = s["table"][q, :-(-m // page)].long()
            if dtype == "bf16":
                into = pool[layer] if name == "k" else pool[layer].transpose(2, 3)
                into[pages[at // page], :, at % page] = mine.to(torch.bfloat16)
                continue
            if dtype == "e2m1":
                held = _exact_values(c, s[name][layer], pages, name)
            else:
                held = (s[name][layer][pages].double() if name == "k" else s[name][layer][pages].double().transpose(2, 3)).transpose(0, 1).reshape(h, -1, d) * scale.view(h, 1, 1)
            held = held[:, :m].transpose(0, 1).clone()
            held[m - n:] = mine
            rows.append(held.reshape(m, h * d))
        out[name] = pool if dtype == "bf16" else torch.cat(rows)
    return out


def _exact_values(c, pool, pages, name):
    """[kv head][token][d] of a row of pages, in 64 bits, nibble by nibble."""
    h, d, page = c["kv_heads"], c["d_head"], c["page"]
    raw = pool[pages].to(torch.int64)
    nibble = torch.stack([raw & 15, raw >> 4], -1)[:, :, :page * d // 2]
    size = nibble & 7
    mantissa, exponent = size & 1, size >> 1
    x = torch.where(exponent > 0, (2 + mantissa).double() * torch.exp2(exponent.double() - 2.0), 0.5 * mantissa.double()) * torch.where(nibble > 7, -1.0, 1.0)
    power = torch.exp2(raw[:, :, page * d // 2:].double() - 127.0)
    if name == "k":
        x = x.reshape(-1, h, page, d // 32, 32) * power.view(-1, h, d // 32, page).permute(0, 1, 3, 2)[..., None]
    else:
        x = x.reshape(-1, h, d // 32, 16, page, 2).permute(0, 1, 4, 2, 5, 3).reshape(-1, h, page, d // 32, 32) * power.view(-1, h, page, d // 32, 1)
    return x.reshape(-1, h, page, d).permute(1, 0, 2, 3).reshape(h, -1, d)


def _exact_decode(c, s):
    h, g, d, page = c["heads"], c["kv_heads"], c["d_head"], c["page"]
    o = torch.zeros(c["n"], h * d, device=DEV, dtype=torch.float64)
    lse = torch.full((c["n"], h), -math.inf, device=DEV, dtype=torch.float64)
    for i, m in enumerate(_lengths(c)):
        if m == 0:
            continue
        pages = s["table"][int(s["seqs"][i]), :-(-m // page)].long()
        k, v = (_exact_values(c, s[x][0], pages, x)[:, :m] for x in ("k", "v"))
        j = torch.arange(m, device=DEV)
        seen = (m - 1 - j < (c["window"] or m)) | (j < c["sinks"])
        x = torch.matmul(s["q"][i].double().view(g, h // g, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
        x = x.masked_fill(~seen, -math.inf)
        lse[i] = torch.logsumexp(x, -1).view(h)
        o[i] = torch.matmul(torch.softmax(x, -1), v).view(h * d)
    return {"o": o, "lse": lse}


def _exact_sample(c, s):
    """Row by row, on the host: the log probability of the token that the random number falls on."""
    t, k, p, f = (x[:, 0].cpu().tolist() for x in _settings(s))
    logits, random, out = s["logits"][:, :c["vocab"]].cpu(), s["random"].cpu().tolist(), []
    for i in range(c["n"]):
        x = logits[i].double()
        left = torch.nonzero(x > -math.inf)[:, 0]
        if len(left) == 0:
            out.append(-math.inf)
            continue
        left = left[torch.argsort(-x[left], stable=True)]          # most probable first, of equal ones the lowest number
        if not t[i] > 0:
            out.append(0.0)
            continue
        if k[i] > 0:
            left = left[:int(k[i])]
        share = torch.softmax(x[left] / t[i], 0)
        if p[i] < 1:
            left = left[:max(1, int((share.cumsum(0) < p[i]).sum()) + 1)]
        z = x[left] / t[i]
        left = left[(z == z[0]) | (torch.exp(z - z[0]) >= f[i])]
        left = torch.sort(left).values
        log = torch.log_softmax(x[left] / t[i], 0)
        at = int((log.exp().cumsum(0) <= random[i]).sum())
        out.append(float(log[min(at, len(left) - 1)]))
    return {"token": None, "logprob": torch.tensor(out, device=DEV, dtype=torch.float64), "kept": None}


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "rope":
        pos, out = _positions(s), {}
        for x in ("q", "k", "dq", "dk"):
            if x in s:
                out[x] = _exact_turn(c, s[x], pos, c["heads"] if "q" in x else c["kv_heads"], -1.0 if x[0] == "d" else 1.0).view(s[x].shape)
        return out
    return {"append": _exact_append, "decode": _exact_decode, "sample": _exact_sample}[c["kind"]](c, s)
