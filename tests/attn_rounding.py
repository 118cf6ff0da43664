"""What the roundings of windowed attention come to, by doing them: probabilities and their gradients to bf16 as operands, results to bf16, all
else in 64 bits.  The norm of the error so made says how far results may be off together, where an element's worst case says little: over
many keys and rows roundings add up like a square root, worst cases one by one.

Bound: 1.1 times that norm.  What the model leaves out are sums in fp32 and exponentials of scores, attn_reference.SLACK of the whole where they
are largest; beside two roundings of 1.65e-3 each in the norm (a half step of 2^-8 of a number's binade is 2.26e-3 of numbers at its
lower end in the root mean square, 1.13e-3 at its upper end), that is sqrt(2 * 1.65^2 + 0.98^2) / sqrt(2 * 1.65^2) = 1.08.  The forward pass
rounds exponentials that are not yet divided by their sum, whose places in their binades are others than the model's: from the least to the
most favourable place a rounding is 2.26 or 1.13 where the mean is 1.65, so o may be 2.26 / 1.65 = 1.37 times the model's."""
import math

import torch

GRADIENTS, FORWARD = 1.1, 1.37

CASES = [
    # batch, queries, keys, heads, kv heads, d, window, sinks
    (1, 300, 300, 2, 1, 64, 0, 0),
    (2, 129, 129, 6, 2, 64, 31, 5),
    (1, 257, 257, 8, 1, 128, 33, 4),
    (2, 70, 31, 4, 2, 64, 12, 2),                 # rows that see nothing
    (1, 100, 517, 4, 1, 128, 130, 7),
    (1, 700, 700, 6, 2, 64, 200, 70),             # from here on also rows that see nothing of a sequence's first keys but the sinks
    (1, 700, 700, 4, 4, 128, 129, 33),
    (3, 391, 391, 4, 2, 64, 100, 100),
    (1, 1500, 1500, 4, 1, 128, 256, 4),           # these rows in eighteen pieces
]


def inputs(seed, rq, rk, n_heads, kv_heads, d):
    g = torch.Generator().manual_seed(seed)
    r = lambda n, w: torch.randn(n, w, generator=g).to(torch.bfloat16)      # noqa: E731
    return r(rq, n_heads * d), r(rk, kv_heads * d), r(rk, kv_heads * d), r(rq, n_heads * d)


def bf16(x):
    return x.to(torch.bfloat16).double()


def head(q, k, v, seen, scale, do=None, o=None, change=None, lost=None):
    """One head as the kernels round it: o, and given do also dq, dk, dv.  o: the stored result that the row term is taken from (None: it is
    taken from the scores).  change, lost: mistakes that a test of the bounds plants, the latter the pairs (row, key) that dk leaves out."""
    s = (q @ k.t() * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[:, None]), 0.0)
    got = {"o": bf16(bf16(p) @ v)}
    if do is not None:
        dp = do @ v.t()
        delta = (p * dp).sum(1, keepdim=True) if o is None else (do * o).sum(1, keepdim=True)
        ds = bf16(p * (dp - delta))
        if change == "no row term":
            ds = bf16(p * dp)
        left = torch.where(lost, 0.0, ds) if lost is not None else ds
        got |= {"dq": bf16(ds @ k * scale), "dk": (left.t() @ q) * scale, "dv": bf16(p).t() @ do}
    return got


def heads(q, k, v, n_heads, kv_heads, d, seen, scale, do=None, o=None, change=None, lost=None):
    """All heads of one sequence, laid out as attn_reference.heads_attention's."""
    group = n_heads // kv_heads
    out = {"o": torch.zeros(q.shape[0], n_heads * d, dtype=torch.float64)}
    if do is not None:
        out |= {"dq": torch.zeros_like(out["o"]), "dk": torch.zeros(k.shape[0], kv_heads * d, dtype=torch.float64), "dv": torch.zeros(k.shape[0], kv_heads * d, dtype=torch.float64)}
    for h in range(n_heads):
        cq, ck = slice(h * d, h * d + d), slice(h // group * d, h // group * d + d)
        a = head(q[:, cq], k[:, ck], v[:, ck], seen, scale, None if do is None else do[:, cq], None if o is None else o[:, cq], change,
                 None if lost is None else lost(h))
        for name, x in a.items():
            out[name][:, cq if name in ("o", "dq") else ck] += x
    for name in ("dk", "dv"):
        if do is not None:
            out[name] = bf16(out[name])
    return out


def assert_near(got, val, model, rows, what):
    """The norm of the error over some rows against the model's."""
    for name, x in model.items():
        r = rows.get(name, slice(None))
        a, b, m = got[name].detach().double().cpu()[r], val[name][r], x[r]
        off, may = float((a - b).norm()), float((m - b).norm()) * (FORWARD if name == "o" else GRADIENTS)
        assert off <= may + 1e-30, (what, name, "relative norms: error %.3g, may be %.3g" % (off / float(b.norm() + 1e-300), may / float(b.norm() + 1e-300)))
