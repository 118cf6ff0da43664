"""Rotations by position, a cache's numbers in 4 bits and the choice of a token, written out from their definitions in 64 bits on the CPU, and a cache
of any format whose every byte is known."""
import math
import random

import numpy as np
import torch

HALF = 2.0 ** -8        # half a step of bf16, relative
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


# ---- rotations -----------------------------------------------------------------------------------------------------
def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, trained=4096.0):
    f = []
    for i in range(rot // 2):
        x = (base * factor ** (rot / (rot - 2)) if scaling == "base" else base) ** (-2.0 * i / rot)
        if scaling == "linear":
            x /= factor
        if scaling == "parts":
            g = min(1.0, max(0.0, (trained * x / (2 * math.pi) - low) / (high - low)))
            x = g * x + (1 - g) * x / factor
        f.append(x)
    return torch.tensor(f, dtype=torch.float64)


def turned(x, pos, f, interleaved, m=1.0, back=False):
    """x [rows][heads][d] in float64, each row turned by its position, and what fp32 sines and products may be off by: a sine or cosine by 2^-22 (its argument and its
    scale rounded once, a polynomial whose last steps round twice), each product and their sum by 2^-24, so 2^-21 of what is added; and the angle, a product of two
    numbers rounded in 64 bits on either side, by 2^-50 of itself."""
    x, r = x.double(), 2 * len(f)
    i, j = (torch.arange(0, r, 2), torch.arange(1, r, 2)) if interleaved else (torch.arange(r // 2), torch.arange(r // 2, r))
    angle = torch.outer(pos.double(), f)[:, None, :]
    c, s = m * angle.cos(), m * angle.sin() * (-1 if back else 1)
    y, off = x.clone(), torch.zeros_like(x)
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    e = abs(m) * (a.abs() + b.abs()) * (2.0 ** -21 + angle.abs() * 2.0 ** -50)
    off[..., i], off[..., j] = e, e
    return y, off


# ---- 4 bits --------------------------------------------------------------------------------------------------------
def to_e2m1(x):
    """Codes (0 .. 15) [..., d] and powers' bytes [..., d / 32] of float64 values, by looking at every power and every value."""
    y = x.double().unflatten(-1, (-1, 32))
    nan = y.isnan().any(-1, keepdim=True)
    big = torch.where(y.isinf(), 3.3895313892515355e38, y.abs()).nan_to_num(0.0)
    top = big.amax(-1, keepdim=True)
    e = torch.full_like(top, 127.0)
    for k in range(126, -128, -1):
        e = torch.where(top <= 7.0 * 2.0 ** k, float(k), e)
    z = y.nan_to_num(0.0, math.inf, -math.inf).abs() / torch.exp2(e)
    best, off = torch.zeros_like(z, dtype=torch.int64), torch.full_like(z, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):              # even mantissas first: in the middle between two they win
        d = (torch.minimum(z, torch.tensor(6.0, dtype=torch.float64)) - GRID[code]).abs()
        best, off = torch.where(d < off, code, best), torch.minimum(d, off)
    code = torch.where(nan, 0, best + 8 * torch.signbit(y).long())
    return code.flatten(-2).to(torch.uint8), torch.where(nan, 255.0, e + 127).squeeze(-1).to(torch.uint8)


def from_e2m1(code, byte):
    x = GRID[(code & 7).long()] * torch.where(code > 7, -1.0, 1.0)
    p = torch.where(byte == 255, math.nan, torch.exp2(byte.double() - 127))
    return (x.unflatten(-1, (-1, 32)) * p[..., None]).flatten(-2)


class Rows:
    """A cache in bf16, e4m3 or e2m1 with pages in no order, on the CPU as codes by token: what the kernels' bytes stand for."""

    def __init__(self, dtype, lens, page, kv_heads=2, d=64, layers=2, slots=None, spare=3, seed=0, wider=1):
        rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
        self.dtype, self.page, self.h, self.d, self.layers, self.lens = dtype, page, kv_heads, d, layers, list(lens)
        need = [-(-m // page) for m in lens]
        self.n_pages, self.ld = sum(need) + spare, max(need) + wider
        order = list(range(self.n_pages))
        rng.shuffle(order)
        self.table, at = [], 0
        for m in need:
            self.table.append(order[at:at + m] + [-1] * (self.ld - m))
            at += m
        self.refs = [1 if p in order[:at] else 0 for p in range(self.n_pages)]
        shape = (layers, self.n_pages, kv_heads, page, d)
        self.scale = {x: (torch.rand(layers, kv_heads, generator=g) + 0.5) / 50 if dtype == "e4m3" else None for x in "kv"}
        self.code, self.power = {}, {}
        for x in "kv":
            y = torch.randn(shape, generator=g)
            if dtype == "e2m1":
                self.code[x], self.power[x] = to_e2m1(y * torch.exp2(torch.randint(-3, 4, shape[:-1] + (1,), generator=g)))
            else:
                self.code[x] = (y * 50).clamp(-448, 448).to(torch.float8_e4m3fn) if dtype == "e4m3" else y.to(torch.bfloat16)

    def raw(self, x):
        """The pool's bytes as the cache's layout has them."""
        c = self.code[x]
        if self.dtype != "e2m1":
            return (c if x == "k" else c.transpose(-1, -2)).contiguous()
        lead = c.shape[:3]
        if x == "k":
            data, power = c[..., 0::2] | (c[..., 1::2] << 4), self.power[x].transpose(-1, -2)
        else:
            y = c.unflatten(-1, (-1, 2, 16))
            data, power = (y[..., 0, :] | (y[..., 1, :] << 4)).flatten(-2).transpose(-1, -2), self.power[x]
        return torch.cat([data.reshape(*lead, -1), power.reshape(*lead, -1)], -1).contiguous()

    def place(self, s, pos):
        p = self.table[s][pos // self.page] if 0 <= pos < self.ld * self.page else -1
        return p if 0 <= p < self.n_pages else -1

    def put(self, x, layer, s, pos, values):
        """values [heads][d] in float64 become token pos of sequence s."""
        p, t = self.place(s, pos), pos % self.page
        if p < 0:
            return
        if self.dtype == "bf16":
            self.code[x][layer, p, :, t] = values.to(torch.bfloat16)
        elif self.dtype == "e4m3":
            y = values / self.scale[x][layer].double()[:, None]
            self.code[x][layer, p, :, t] = torch.where(y.isnan(), y, y.clamp(-448, 448)).to(torch.float8_e4m3fn)
        else:
            self.code[x][layer, p, :, t], self.power[x][layer, p, :, t] = to_e2m1(values)

    def get(self, x, layer, s, pos):
        """[heads][d] in float64, or None where there is no such token."""
        p, t = self.place(s, pos) if 0 <= pos < self.lens[s] else -1, pos % self.page
        if p < 0:
            return None
        c = self.code[x][layer, p, :, t]
        if self.dtype == "e2m1":
            return from_e2m1(c, self.power[x][layer, p, :, t])
        return c.double() if self.dtype == "bf16" else c.double() * self.scale[x][layer].double()[:, None]

    def on(self, S, dev):
        """The cache on a device (its tensors are kept here)."""
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)      # noqa: E731
        self.t = dict(k=self.raw("k").to(dev), v=self.raw("v").to(dev), table=i32(self.table), lengths=i32(self.lens), refs=i32(self.refs),
                      k_scale=None if self.scale["k"] is None else self.scale["k"].to(dev), v_scale=None if self.scale["v"] is None else self.scale["v"].to(dev))
        kind = {"bf16": S.SIF_BF16, "e4m3": S.SIF_E4M3, "e2m1": S.SIF_E2M1}[self.dtype]
        self.cache = S.kv_cache(**self.t, dtype=kind, page_tokens=self.page)
        return self.cache

    def check(self, what=""):
        """Every byte of the device's pools (of NaN only that it is one)."""
        for x in "kv":
            got, want = self.t[x].cpu(), self.raw(x)
            both = torch.zeros(got.shape, dtype=torch.bool) if self.dtype == "e2m1" else got.float().isnan() & want.float().isnan()
            bits = torch.int16 if self.dtype == "bf16" else torch.uint8
            bad = torch.nonzero((got.view(bits) != want.view(bits)) & ~both)
            assert len(bad) == 0, (what, x, len(bad), bad[:4].tolist())


# ---- tokens --------------------------------------------------------------------------------------------------------
def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log probability, tokens left) of one row, logits as float64 numbers, by the limits' definitions."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    if (x == np.inf).any():
        x = np.where(x == np.inf, 0.0, -np.inf)
    order = [int(i) for i in np.argsort(-x, kind="stable") if x[i] > -np.inf]
    if not order:
        return -1, -math.inf, 0
    if not temperature > 0:
        return order[0], 0.0, 1
    if top_k > 0:
        order = order[:top_k]
    top = x[order[0]]
    with np.errstate(over="ignore", invalid="ignore"):
        z = np.where(x[order] == top, 0.0, (x[order] - top) / temperature)
        w = np.where(np.isnan(z), 0.0, np.exp(z))
    if top_p < 1:
        n, total, goal = 0, 0.0, top_p * w.sum()
        while n == 0 or (n < len(order) and total < goal):
            total += w[n]
            n += 1
        order, w = order[:n], w[:n]
    if min_p > 0:
        n = max(1, int((w >= min(min_p, 1.0)).sum()))
        order, w = order[:n], w[:n]
    left = sorted(zip(order, w))
    goal, total = min(max(u, 0.0) if u == u else 0.0, 1 - 2.0 ** -24) * w.sum(), 0.0
    # the sums are of whole numbers w 2^s, s the largest up to 51 with which `vocab` of them stay within 2^62: less than half of one is nothing, which shows at u = 0
    least = 2.0 ** -(1 + min(51, 62 - math.ceil(math.log2(len(x)))))
    for i, share in left:
        total += share if share > least else 0.0
        if total > goal:
            return i, math.log(share / w.sum()) if share > 0 else -math.inf, len(left)
    raise AssertionError("no token")
