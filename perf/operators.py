"""Attention with a sliding window and sinks, attention of new tokens over a paged cache, and the cache's page operations,
as cases that can be timed and compared.

Three kinds of pass, as a program on this library makes them (`own`), and the same in elementary torch operations:

  window   attention of whole sequences under a causal mask with a window of recent keys and a few first keys (sinks) that
           stay visible: forward, or forward and backward as a training step does
  decode   attention of one new token per sequence over a paged key-value cache
  pages    operations on the pages of such a cache: a round of forked sequences (free, fork, extend, write), compaction,
           plain page copies

Layouts: rows of q, k, v and o are tokens, a head is a column slice.  A cache holds keys as [layer][page][kv head][token][d] and
values as [layer][page][kv head][d][token], the page table [sequence][page], the sequences' lengths and the pages' reference
counts.  Head counts and sizes are those of the configurations in synth_inputs.py and perf/cases.py, or generic ones.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---- cases -------------------------------------------------------------------------------------------------------
def _window(**kw):
    return dict(dict(kind="window", train=True, batch=1, packed=False), **kw)


def _decode(**kw):
    return dict(dict(kind="decode", dtype="bf16", window=0, sinks=0), **kw)


def listed():
    return [
        # the small decoder's training step: nothing but latency
        _window(name="window_tiny", batch=4, seq_q=64, seq_k=64, heads=4, kv_heads=2, d_head=64, window=16, sinks=2),
        # documents of 1 to 611 tokens laid back to back, heads of 64, nothing on a tile boundary
        _window(name="window_packed", packed=True, batch=9, seq_q=611, seq_k=611, heads=12, kv_heads=4, d_head=64, window=100, sinks=3),
        # a pipeline stage's attention with as many key heads as query heads
        _window(name="window_stage", batch=2, seq_q=2048, seq_k=2048, heads=16, kv_heads=16, d_head=128, window=512, sinks=4),
        # training on long sequences, four query heads to a key head
        _window(name="window_long", batch=1, seq_q=8192, seq_k=8192, heads=16, kv_heads=4, d_head=128, window=1024, sinks=4),
        # a prompt's next piece behind what the cache already holds, inference only
        _window(name="window_piece", train=False, batch=2, seq_q=500, seq_k=8191, heads=32, kv_heads=8, d_head=128, window=4096, sinks=16),
        # one request of odd length at an idle instance: latency
        _decode(name="decode_one", n=1, len_min=77, len_max=77, heads=12, kv_heads=12, d_head=64, page=16),
        # a full batch of requests of very different lengths
        _decode(name="decode_batch", n=64, len_min=1, len_max=8192, heads=32, kv_heads=8, d_head=128, page=16),
        # one very long context: too few rows for the chip, so the length has to be split
        _decode(name="decode_long", n=1, len_min=262011, len_max=262011, heads=32, kv_heads=8, d_head=128, page=64),
        # many requests under a window with sinks, the cache in 8 bits
        _decode(name="decode_window_8bit", dtype="e4m3", n=128, len_min=100, len_max=16384, heads=16, kv_heads=2, d_head=128, page=32, window=1024, sinks=4),
        # four sequences, each forked once, a few tokens on: latency
        dict(name="pages_round_small", kind="round", dtype="bf16", layers=2, n=4, forks=1, len_min=5, len_max=300, grow=3, kv_heads=4, d_head=64, page=16),
        # sampling of several answers to each of 32 prompts over a cache of twelve layers: shared pages are copied when written to
        dict(name="pages_round", kind="round", dtype="bf16", layers=12, n=32, forks=4, len_min=30, len_max=2000, grow=9, kv_heads=8, d_head=128, page=16),
        # a cache in which a third of the sequences have ended is put together again
        dict(name="pages_compact", kind="compact", dtype="bf16", layers=8, n=96, len_min=100, len_max=1500, kv_heads=8, d_head=128, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    kv = rng.choice([h for h in (1, 2, 4, 8, 12, 16) if h <= most])
    return dict(heads=kv * rng.choice([g for g in (1, 2, 3, 4, 8) if kv * g <= most]), kv_heads=kv, d_head=rng.choice((64, 128)))


def _draw(rng):
    pick = rng.random()
    if pick < 0.5:
        c = dict(train=rng.random() < 0.7, window=_log(rng, 8, 4096), sinks=rng.choice((0, 1, 4, rng.randint(2, 64))), **_heads(rng, 16))
        s = _log(rng, 24, 6000)
        if rng.random() < 0.3:
            return _window(packed=True, batch=rng.randint(2, 12), seq_q=min(s, 900), seq_k=min(s, 900), **c)
        if c["train"] or rng.random() < 0.5:
            return _window(batch=rng.randint(1, 3), seq_q=s, seq_k=s, **c)
        return _window(batch=rng.randint(1, 3), seq_q=_log(rng, 2, 1000), seq_k=1000 + s, **c)
    if pick < 0.82:
        lo = _log(rng, 1, 4000)
        window = rng.choice((0, _log(rng, 16, 4096)))
        return _decode(dtype=rng.choice(("bf16", "e4m3")), n=_log(rng, 1, 128), len_min=lo, len_max=lo + _log(rng, 1, 60000), page=rng.choice((16, 32, 64, 128)),
                       window=window, sinks=rng.choice((0, 4, 33)) if window else 0, **_heads(rng, 48))
    c = dict(dtype=rng.choice(("bf16", "e4m3")), layers=rng.randint(1, 12), n=_log(rng, 2, 64), len_min=rng.randint(1, 200), kv_heads=rng.choice((1, 2, 4, 8, 12)),
             d_head=rng.choice((64, 128)), page=rng.choice((16, 32, 64)))
    c["len_max"] = c["len_min"] + _log(rng, 10, 1500)
    if rng.random() < 0.6:
        return dict(kind="round", forks=rng.randint(1, 6), grow=rng.randint(1, 40), **c)
    return dict(kind="compact", **c)


def _cost(c):
    """What the plain form holds at once, in bytes."""
    if c["kind"] == "window":
        rows = (sum(_lengths(c)), sum(_lengths(c))) if c["packed"] else (c["batch"] * c["seq_q"], c["seq_k"])
        return 4.0 * c["heads"] * rows[0] * rows[1]
    if c["kind"] == "decode":
        return 8.0 * c["n"] * c["len_max"] * c["kv_heads"] * c["d_head"]
    return 4.0 * _pool(c)["n_pages"] * c["layers"] * c["kv_heads"] * c["page"] * c["d_head"]


def draw(rng):
    listings = listed()
    while True:
        c = _draw(rng)
        alike = [x for x in listings if x["kind"] == c["kind"]]
        if _cost(c) <= max(_cost(x) for x in alike) and work(c)["flops"] <= max(work(x)["flops"] for x in alike) and work(c)["bytes"] <= max(work(x)["bytes"] for x in alike):
            return c


# ---- shapes, and the work a pass cannot do without ----------------------------------------------------------------
def _lengths(c):
    """The sequences' lengths: spread over the case's range, in no order."""
    if c["kind"] == "window":
        n, lo, hi = c["batch"], 1, c["seq_q"]
    else:
        n, lo, hi = c["n"], c["len_min"], c["len_max"]
    if n == 1:
        return [hi]
    got = [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return [got[i * 7 % n] for i in range(n)] if n % 7 else got[::-1]


def _bits(c):
    return 1 if c.get("dtype") == "e4m3" else 2


def _pool(c):
    """Pages, table width and sequences of a `round` or `compact` case."""
    grow, forks = c.get("grow", 0), c.get("forks", 0)
    width = -(-(max(_lengths(c)) + grow) // c["page"])
    used = sum(-(-m // c["page"]) for m in _lengths(c))
    more = c["n"] * forks * (grow // c["page"] + 2)
    return {"width": width, "n_pages": used + more + 5, "n_seqs": c["n"] * (1 + forks)}


def _pairs(sq, sk, window, sinks):
    """Keys that are visible to the rows of one sequence."""
    first = sk - sq
    total = 0
    for p in range(max(first, 0), sk):
        near = min(p + 1, window) if window else p + 1
        total += near + min(sinks, p + 1 - near)
    return total


def work(c):
    """Every input and output once; the two products of attention over visible keys (backward: five)."""
    if c["kind"] == "window":
        lens = [(m, m) for m in _lengths(c)] if c["packed"] else [(c["seq_q"], c["seq_k"])]
        times = 1 if c["packed"] else c["batch"]
        pairs = times * sum(_pairs(a, b, c["window"], c["sinks"]) for a, b in lens)
        rq, rk = times * sum(a for a, _ in lens), times * sum(b for _, b in lens)
        q, k = 2.0 * rq * c["heads"] * c["d_head"], 2.0 * rk * c["kv_heads"] * c["d_head"]
        lse = 4.0 * rq * c["heads"]
        if c["train"]:
            return {"bytes": 4 * q + 4 * k + lse, "flops": 14.0 * pairs * c["heads"] * c["d_head"]}
        return {"bytes": 2 * q + 2 * k + lse, "flops": 4.0 * pairs * c["heads"] * c["d_head"]}
    if c["kind"] == "decode":
        seen = sum(_pairs(1, m, c["window"], c["sinks"]) for m in _lengths(c))
        return {"bytes": 2.0 * _bits(c) * seen * c["kv_heads"] * c["d_head"] + 4.0 * c["n"] * c["heads"] * c["d_head"], "flops": 4.0 * seen * c["heads"] * c["d_head"]}
    page = 2.0 * _bits(c) * c["layers"] * c["kv_heads"] * c["page"] * c["d_head"]
    if c["kind"] == "compact":
        return {"bytes": 2 * page * len(_moves(c)) + 4.0 * _pool(c)["n_pages"], "flops": 0.0}
    lens = _lengths(c)
    shared = sum(c["forks"] for m in lens if m % c["page"])
    table = 8.0 * c["forks"] * sum(-(-m // c["page"]) for m in lens)
    rows = c["n"] * c["forks"] * c["grow"] * c["kv_heads"] * c["d_head"]
    return {"bytes": 2 * page * shared + table + (4.0 + 2.0 * _bits(c)) * rows, "flops": 0.0}


def _left(c):
    """A compact case's sequences that go on: two of three."""
    return [i for i in range(c["n"]) if i % 3 != 1]


def _moves(c):
    """How many pages change their place at most: as many as the ended sequences held, or as go on, whichever is less."""
    lens = _lengths(c)
    stay = sum(-(-lens[i] // c["page"]) for i in _left(c))
    n_pages = _pool(c)["n_pages"]
    return range(int(stay * (1 - stay / n_pages)))


# ---- states ------------------------------------------------------------------------------------------------------
def _bf16(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _page_data(gen, c, layers, n_pages):
    """Keys and values of a cache, and in 8 bits the scales that go with them (a value is what is held times its scale)."""
    def some(*shape):
        x = torch.empty(shape, device=DEV, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float8_e4m3fn)
        for part in x.view(-1).split(1 << 27):
            y = torch.randn(part.numel(), generator=gen, device=DEV, dtype=torch.float32)
            part.copy_(y if c["dtype"] == "bf16" else (y * 64.0).clamp(-448.0, 448.0))
        return x
    k = some(layers, n_pages, c["kv_heads"], c["page"], c["d_head"])
    v = some(layers, n_pages, c["kv_heads"], c["d_head"], c["page"])
    scale = lambda: (0.8 + 0.4 * torch.rand(layers, c["kv_heads"], generator=gen, device=DEV)) / 64.0      # noqa: E731
    return dict(k=k, v=v, k_scale=scale() if c["dtype"] == "e4m3" else None, v_scale=scale() if c["dtype"] == "e4m3" else None)


def _tables(gen, lens, n_seqs, width, n_pages, page):
    """The first len(lens) of n_seqs sequences hold pages of a shuffled pool, the others are empty."""
    count = torch.tensor([-(-m // page) for m in lens] + [0] * (n_seqs - len(lens)), device=DEV)
    slot = torch.arange(width, device=DEV)[None, :].expand(n_seqs, width)
    here = slot < count[:, None]
    first = (count.cumsum(0) - count)[:, None]
    order = torch.randperm(n_pages, generator=gen, device=DEV)
    table = torch.where(here, order[(first + slot).clamp(max=n_pages - 1)], torch.full_like(slot, -1)).to(torch.int32).contiguous()
    refs = torch.zeros(n_pages, device=DEV, dtype=torch.int32)
    refs[order[:int(count.sum())]] = 1
    return table, torch.tensor(list(lens) + [0] * (n_seqs - len(lens)), device=DEV, dtype=torch.int32), refs


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "window":
        h, g, d = c["heads"], c["kv_heads"], c["d_head"]
        lens = _lengths(c) if c["packed"] else [c["seq_q"]] * c["batch"]
        rq = sum(lens)
        rk = rq if c["packed"] else c["batch"] * c["seq_k"]
        s |= dict(q=_bf16(gen, rq, h * d), k=_bf16(gen, rk, g * d), v=_bf16(gen, rk, g * d))
        s |= dict(o=torch.empty_like(s["q"]), lse=torch.empty(h, rq, device=DEV))
        if c["train"]:
            s |= dict(do=_bf16(gen, rq, h * d), dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]))
        if c["packed"]:
            s["starts"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device=DEV, dtype=torch.int32)
        return s
    lens = _lengths(c)
    if c["kind"] == "decode":
        width = -(-max(lens) // c["page"])
        n_pages = sum(-(-m // c["page"]) for m in lens) + 3
        s |= _page_data(gen, c, 1, n_pages)
        s["table"], s["lengths"], s["refs"] = _tables(gen, lens, c["n"], width, n_pages, c["page"])
        s["q"] = _bf16(gen, c["n"], c["heads"] * c["d_head"])
        s |= dict(o=torch.empty_like(s["q"]), lse=torch.empty(c["n"], c["heads"], device=DEV))
        return s
    p = _pool(c)
    s |= _page_data(gen, c, c["layers"], p["n_pages"])
    s["table"], s["lengths"], s["refs"] = _tables(gen, lens, p["n_seqs"], p["width"], p["n_pages"], c["page"])
    if c["kind"] == "round":
        n, f = c["n"], c["forks"]
        s["src"] = torch.arange(n, device=DEV, dtype=torch.int32).repeat_interleave(f).contiguous()
        s["dst"] = torch.arange(n, n + n * f, device=DEV, dtype=torch.int32)
        s["counts"] = torch.full((n * f,), c["grow"], device=DEV, dtype=torch.int32)
        s["starts"] = torch.arange(0, (n * f + 1) * c["grow"], c["grow"], device=DEV, dtype=torch.int32)
        s["k_new"] = _bf16(gen, n * f * c["grow"], c["kv_heads"] * c["d_head"])
        s["v_new"] = _bf16(gen, n * f * c["grow"], c["kv_heads"] * c["d_head"])
        s["status"] = torch.zeros(n * f, device=DEV, dtype=torch.int32)
    else:
        ended = torch.tensor([i for i in range(c["n"]) if i not in set(_left(c))], device=DEV)
        gone = s["table"][ended]
        s["refs"][gone[gone >= 0].long()] = 0
        s["table"][ended] = -1
        s["lengths"][ended] = 0
        s |= dict(table0=s["table"].clone(), refs0=s["refs"].clone())
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _seen(qpos, kpos, window, sinks):
    """Whether the key at kpos is visible to the query at qpos."""
    near = (kpos > qpos - window) if window else torch.ones_like(kpos <= qpos)
    return (kpos <= qpos) & (near | (kpos < sinks))


def _softmax(s, seen):
    """Probabilities and log sum exp of masked scores; rows that see nothing have zeros and -inf."""
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return p / torch.where(total > 0, total, 1.0), lse


def _plain_window(s):
    c = s["case"]
    h, g, d, w = c["heads"], c["kv_heads"], c["d_head"], c["window"]
    b, n = (1, h // g) if c["packed"] else (c["batch"], h // g)
    rq, rk = s["q"].shape[0] // b, s["k"].shape[0] // b
    if c["packed"]:
        row = torch.arange(rq, device=DEV)
        seq = torch.searchsorted(s["starts"], row.to(torch.int32), right=True) - 1
        pos = row - s["starts"].long()[seq]
        seen = _seen(pos[:, None], pos[None, :], w, c["sinks"]) & (seq[:, None] == seq[None, :])
    else:
        seen = _seen(torch.arange(rq, device=DEV)[:, None] + (rk - rq), torch.arange(rk, device=DEV)[None, :], w, c["sinks"])
    # queries as [batch][key head][query head of it, row][d]
    of_q = lambda x: x.float().view(b, rq, g, n, d).permute(0, 2, 3, 1, 4).reshape(b, g, n * rq, d)      # noqa: E731
    of_k = lambda x: x.float().view(b, rk, g, d).permute(0, 2, 1, 3).contiguous()      # noqa: E731
    to_q = lambda x: x.view(b, g, n, rq, d).permute(0, 3, 1, 2, 4).reshape(b * rq, h * d).to(torch.bfloat16)      # noqa: E731
    to_k = lambda x: x.permute(0, 2, 1, 3).reshape(b * rk, g * d).to(torch.bfloat16)      # noqa: E731
    q, k, v, scale = of_q(s["q"]), of_k(s["k"]), of_k(s["v"]), 1.0 / math.sqrt(d)
    seen = seen.repeat(n, 1)
    p, lse = _softmax(torch.matmul(q, k.transpose(2, 3).contiguous()) * scale, seen)
    out = {"o": to_q(torch.matmul(p, v)), "lse": lse.view(b, g * n, rq).transpose(0, 1).reshape(h, b * rq)}
    if not c["train"]:
        return out
    do = of_q(s["do"])
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    return out | {"dq": to_q(torch.matmul(ds, k)), "dk": to_k(torch.matmul(ds.transpose(2, 3).contiguous(), q)), "dv": to_k(dv)}


def _plain_decode(s):
    c = s["case"]
    n, h, g, d = c["n"], c["heads"], c["kv_heads"], c["d_head"]
    page = s["table"].long().clamp(min=0)
    k = s["k"][0][page].permute(0, 2, 1, 3, 4).reshape(n, g, -1, d).float()
    v = s["v"][0][page].permute(0, 2, 1, 4, 3).reshape(n, g, -1, d).float()
    if c["dtype"] == "e4m3":
        k, v = k * s["k_scale"][0][None, :, None, None], v * s["v_scale"][0][None, :, None, None]
    last = s["lengths"].long()[:, None] - 1
    seen = _seen(last, torch.arange(k.shape[2], device=DEV)[None, :], c["window"], c["sinks"])[:, None, None, :]
    q = s["q"].float().view(n, g, h // g, d)
    p, lse = _softmax(torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d), seen)
    return {"o": torch.matmul(p, v).reshape(n, h * d).to(torch.bfloat16), "lse": lse.reshape(n, h)}


def _values(x):
    """What is held in 8 bits as the values it stands for."""
    return x if x.dtype == torch.bfloat16 else x.to(torch.bfloat16)


def _plain_round(s):
    c = s["case"]
    table, lengths, refs, page, grow = s["table"], s["lengths"], s["refs"], c["page"], c["grow"]
    src, dst = s["src"].long(), s["dst"].long()
    # free: the pages of the sequences lose a reference
    old = table[dst].long()
    refs.index_add_(0, old.clamp(min=0).view(-1), -(old >= 0).to(torch.int32).view(-1))
    # fork: the new sequences share the pages of the old ones
    rows = table[src]
    refs.index_add_(0, rows.long().clamp(min=0).view(-1), (rows >= 0).to(torch.int32).view(-1))
    # extend: new pages for the tokens to come, the lowest free ones in the order of the sequences; a last page that is
    # shared and not full is copied first
    m = lengths[src].long()
    counts = s["counts"].long()
    before, after = (m + page - 1) // page, (m + counts + page - 1) // page
    last = torch.gather(rows, 1, (before - 1).clamp(min=0)[:, None])[:, 0].long()
    copied = (m % page != 0) & (refs[last.clamp(min=0)] > 1)
    need = after - before + copied
    first = need.cumsum(0) - need
    lowest = torch.argsort((refs > 0).to(torch.int8), stable=True)
    slot = torch.arange(table.shape[1], device=DEV)[None, :]
    begin = (before - copied.long())[:, None]
    fresh = (slot >= begin) & (slot < after[:, None])
    new = lowest[(first[:, None] + slot - begin).clamp(0, refs.shape[0] - 1)]
    rows = torch.where(fresh, new.to(torch.int32), rows)
    refs.index_add_(0, new.reshape(-1), fresh.to(torch.int32).reshape(-1))
    refs.index_add_(0, last.clamp(min=0), -copied.to(torch.int32))
    to = torch.where(copied, torch.gather(rows, 1, (before - 1).clamp(min=0)[:, None])[:, 0].long(), last.clamp(min=0))
    raw = (lambda x: x) if c["dtype"] == "bf16" else (lambda x: x.view(torch.uint8))
    raw(s["k"])[:, to] = raw(s["k"])[:, last.clamp(min=0)]
    raw(s["v"])[:, to] = raw(s["v"])[:, last.clamp(min=0)]
    table[dst] = rows
    lengths[dst] = (m + counts).to(torch.int32)
    # write: the new tokens' keys and values of one layer
    layer, g, d = c["layers"] - 1, c["kv_heads"], c["d_head"]
    pos = m[:, None] + torch.arange(grow, device=DEV)[None, :]
    at = torch.gather(rows.long(), 1, pos // page).view(-1)
    off = (pos % page).view(-1)
    k, v = s["k_new"].view(-1, g, d), s["v_new"].view(-1, g, d)
    if c["dtype"] == "e4m3":
        held = lambda x, scale: (x.float() / scale[layer][None, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)      # noqa: E731
        k, v = held(k, s["k_scale"]).view(torch.uint8), held(v, s["v_scale"]).view(torch.uint8)
    raw(s["k"])[layer].permute(0, 2, 1, 3)[at, off] = k
    raw(s["v"])[layer].permute(0, 3, 1, 2)[at, off] = v
    s["status"].zero_()
    return _round_outputs(s)


def _round_outputs(s):
    return {"table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "status": s["status"], "k": _values(s["k"]), "v": _values(s["v"])}


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    table, refs = s["table"], s["refs"]
    used = refs > 0
    total = used.sum()
    number = torch.arange(refs.shape[0], device=DEV)
    # the k-th used page from `total` on goes to the k-th free page below it
    moved, hole = used & (number >= total), ~used & (number < total)
    holes = torch.argsort((~hole).to(torch.int8), stable=True)
    to = torch.where(moved, holes[(moved.long().cumsum(0) - 1).clamp(min=0)], number)
    # every page asks where its contents come from (itself, if nothing moves there)
    source = torch.cat([number, number[:1]]).scatter(0, torch.where(moved, to, number.shape[0]), number)[:-1]
    raw = (lambda x: x) if s["case"]["dtype"] == "bf16" else (lambda x: x.view(torch.uint8))
    raw(s["k"]).copy_(raw(s["k"])[:, source])
    raw(s["v"]).copy_(raw(s["v"])[:, source])
    table.copy_(torch.where(table >= 0, to[table.long().clamp(min=0)].to(torch.int32), table))
    refs.copy_(torch.where(moved, 0, refs[source]))
    return {"table": table, "refs": refs, "k": _values(s["k"]), "v": _values(s["v"])}


# ---- the library's calls -----------------------------------------------------------------------------------------
def _handles(s):
    """What a program sets up once for its buffers: argument structures and workspaces."""
    import paper_2503_02550_amd as S
    c = s["case"]
    if c["kind"] == "window":
        a = S.window_attn_args(s["q"], s["k"], s["v"], s["o"], heads=c["heads"], kv_heads=c["kv_heads"], d_head=c["d_head"], batch=c["batch"], seq_q=c["seq_q"],
                               seq_k=c["seq_k"], window=c["window"], sinks=c["sinks"], lse=s["lse"], starts=s.get("starts"), rows=s["q"].shape[0],
                               d_o=s.get("do"), dq=s.get("dq"), dk=s.get("dk"), dv=s.get("dv"))
        if c["train"]:
            n = S.sif_window_attn_bwd_workspace_bytes(a)
            s["workspace"] = torch.empty(n, device=DEV, dtype=torch.uint8)
            S.set_workspace(a, s["workspace"], n)
        return S, a
    cache = S.kv_cache(s["k"], s["v"], s["table"], s["lengths"], s["refs"], dtype=S.SIF_BF16 if c["dtype"] == "bf16" else S.SIF_E4M3, page_tokens=c["page"],
                       k_scale=s["k_scale"], v_scale=s["v_scale"])
    if c["kind"] == "decode":
        a = S.attn_decode_args(s["q"], s["o"], n=c["n"], heads=c["heads"], window=c["window"], sinks=c["sinks"], max_tokens=c["len_max"], lse=s["lse"])
        n = S.sif_attn_decode_workspace_bytes(cache, a)
        s["workspace"] = torch.empty(n, device=DEV, dtype=torch.uint8)
        S.set_workspace(a, s["workspace"], n)
        return S, cache, a
    n = S.sif_kv_workspace_bytes(cache)
    s["workspace"] = torch.empty(n, device=DEV, dtype=torch.uint8)
    return S, cache, n


def _own(s):
    c = s["case"]
    if "handles" not in s:
        s["handles"] = _handles(s)
    if c["kind"] == "window":
        S, a = s["handles"]
        S.sif_k_window_attn_fwd(a)
        if not c["train"]:
            return {"o": s["o"], "lse": s["lse"]}
        S.sif_k_window_attn_bwd(a)
        return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if c["kind"] == "decode":
        S, cache, a = s["handles"]
        S.sif_k_attn_decode(cache, a)
        return {"o": s["o"], "lse": s["lse"]}
    S, cache, n = s["handles"]
    if c["kind"] == "round":
        m = s["dst"].shape[0]
        S.sif_k_kv_free(cache, s["dst"], m)
        S.sif_k_kv_fork(cache, s["src"], s["dst"], m)
        S.sif_k_kv_extend(cache, s["dst"], s["counts"], m, s["workspace"], n, status=s["status"])
        S.sif_k_kv_write(cache, c["layers"] - 1, s["k_new"], s["v_new"], s["dst"], m, starts=s["starts"], rows=s["k_new"].shape[0])
        return _round_outputs(s)
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    S.sif_k_kv_compact(cache, s["workspace"], n)
    return {"table": s["table"], "refs": s["refs"], "k": _values(s["k"]), "v": _values(s["v"])}


def run(s):
    if own:
        return _own(s)
    return {"window": _plain_window, "decode": _plain_decode, "round": _plain_round, "compact": _plain_compact}[s["case"]["kind"]](s)


# ---- the same in 64 bits -----------------------------------------------------------------------------------------
def _exact_attention(q, k, v, seen):
    """[rows][d] of one head, from the definition, with autograd for what comes after."""
    s = q @ k.t() / math.sqrt(q.shape[1])
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1)
    w = torch.where(seen, (s - torch.where(lse > -math.inf, lse, 0.0)[:, None]).exp(), 0.0)
    return w @ v, lse.detach()


def _exact_mask(first, sq, sk, window, sinks):
    i = torch.arange(first, first + sq, device=DEV).view(-1, 1)
    j = torch.arange(sk, device=DEV).view(1, -1)
    return (j <= i) & ((i - j < (window if window else 1 << 40)) | (j < sinks))


def _exact_window(c, s):
    h, g, d = c["heads"], c["kv_heads"], c["d_head"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    out = {"o": torch.zeros_like(q), "lse": torch.full((h, q.shape[0]), -math.inf, device=DEV, dtype=torch.float64)}
    if c["train"]:
        do = s["do"].double()
        out |= {"dq": torch.zeros_like(q), "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    lens = _lengths(c) if c["packed"] else [c["seq_q"]] * c["batch"]
    a0 = b0 = 0
    for m in lens:
        sk = m if c["packed"] else c["seq_k"]
        seen = _exact_mask(sk - m, m, sk, c["window"], c["sinks"])
        rows, keys = slice(a0, a0 + m), slice(b0, b0 + sk)
        for head in range(h):
            cq, ck = slice(head * d, head * d + d), slice(head // (h // g) * d, head // (h // g) * d + d)
            x = [q[rows, cq].detach().requires_grad_(c["train"]), k[keys, ck].detach().requires_grad_(c["train"]), v[keys, ck].detach().requires_grad_(c["train"])]
            o, lse = _exact_attention(*x, seen)
            out["o"][rows, cq], out["lse"][head, rows] = o.detach(), lse
            if c["train"]:
                dq, dk, dv = torch.autograd.grad(o, x, do[rows, cq])
                out["dq"][rows, cq] = dq
                out["dk"][keys, ck] += dk
                out["dv"][keys, ck] += dv
        a0, b0 = a0 + m, b0 + sk
    return out


def _exact_decode(c, s):
    h, g, d, page = c["heads"], c["kv_heads"], c["d_head"], c["page"]
    o = torch.zeros(c["n"], h * d, device=DEV, dtype=torch.float64)
    lse = torch.full((c["n"], h), -math.inf, device=DEV, dtype=torch.float64)
    for i, m in enumerate(_lengths(c)):
        at = s["table"][i, :-(-m // page)].long()
        seen = _exact_mask(m - 1, 1, m, c["window"], c["sinks"])
        for kv in range(g):
            k = s["k"][0, at, kv].double().reshape(-1, d)[:m]
            v = s["v"][0, at, kv].double().transpose(1, 2).reshape(-1, d)[:m]
            if c["dtype"] == "e4m3":
                k, v = k * s["k_scale"][0, kv].double(), v * s["v_scale"][0, kv].double()
            q = s["q"][i].double().view(g, h // g, d)[kv]
            a, b = _exact_attention(q, k, v, seen.expand(h // g, m))
            o[i].view(g, h // g, d)[kv], lse[i].view(g, h // g)[kv] = a, b
    return {"o": o, "lse": lse}


def _exact_round(c, s):
    """One sequence after the other, as the operations are defined."""
    page, grow = c["page"], c["grow"]
    table, refs = s["table"].cpu().tolist(), s["refs"].cpu().tolist()
    k, v = (s[x].clone() if c["dtype"] == "bf16" else s[x].to(torch.bfloat16) for x in ("k", "v"))
    lens = s["lengths"].cpu().tolist()
    pairs = list(zip(s["src"].cpu().tolist(), s["dst"].cpu().tolist()))
    for a, b in pairs:
        for p in table[a]:
            if p >= 0:
                refs[p] += 1
        table[b], lens[b] = list(table[a]), lens[a]
    stood, empty = list(refs), [p for p, r in enumerate(refs) if r <= 0]
    empty.reverse()
    moved = []
    for _, b in pairs:
        m = lens[b]
        if m % page and stood[table[b][m // page]] > 1:
            p = empty.pop()
            moved.append((table[b][m // page], p))
            refs[table[b][m // page]] -= 1
            refs[p] += 1
            table[b][m // page] = p
        for j in range(-(-m // page), -(-(m + grow) // page)):
            table[b][j] = empty.pop()
            refs[table[b][j]] += 1
        lens[b] = m + grow
    if moved:
        x, y = torch.tensor(moved, device=DEV).t()
        k[:, y], v[:, y] = k[:, x], v[:, x]
    layer, g, d = c["layers"] - 1, c["kv_heads"], c["d_head"]
    place = torch.tensor([(table[b][p // page], p % page) for _, b in pairs for p in range(lens[b] - grow, lens[b])], device=DEV)
    for pool, name, scale in ((k, "k_new", s["k_scale"]), (v, "v_new", s["v_scale"])):
        x = s[name].double().view(-1, g, d)
        if c["dtype"] == "e4m3":
            x = (s[name].float().view(-1, g, d) / scale[layer].view(1, g, 1)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).double()
        into = pool[layer].transpose(1, 2) if name == "k_new" else pool[layer].permute(0, 3, 1, 2)
        into[place[:, 0], place[:, 1]] = x.to(torch.bfloat16)
    return {"table": None, "lengths": None, "refs": None, "status": None, "k": k, "v": v}


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "window":
        return _exact_window(c, s)
    if c["kind"] == "decode":
        return _exact_decode(c, s)
    if c["kind"] == "round":
        return _exact_round(c, s)
    # compaction: the lowest pages take what the highest hold
    refs = s["refs"].cpu().tolist()
    total = sum(r > 0 for r in refs)
    to = [p for p in range(total) if refs[p] <= 0]
    of = [p for p in range(total, len(refs)) if refs[p] > 0]
    k, v = (s[x] if c["dtype"] == "bf16" else s[x].to(torch.bfloat16) for x in ("k", "v"))
    if to:
        x, y = torch.tensor(of, device=DEV), torch.tensor(to, device=DEV)
        k[:, y], v[:, y] = k[:, x], v[:, x]
    return {"table": None, "refs": None, "k": k, "v": v}
