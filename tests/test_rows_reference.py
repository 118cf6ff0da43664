"""The reference of rotations and 4-bit numbers against themselves, and the table of a rotation (a pure host function) against its formulas."""
import math

import pytest
import torch

import paper_2503_02550_amd as S
from rows_reference import Rows, frequencies, from_e2m1, sample, to_e2m1, turned

HOW = {"plain": S.SIF_ROPE_PLAIN, "linear": S.SIF_ROPE_LINEAR, "base": S.SIF_ROPE_BASE, "parts": S.SIF_ROPE_PARTS}


@pytest.mark.parametrize("rot", [16, 48, 64, 128, 256])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0), dict(scaling="base", factor=0.5),
                                dict(scaling="parts", factor=32.0, low=1.0, high=4.0, trained=8192.0), dict(scaling="parts", factor=3.0, low=-2.0, high=32.0, trained=100.0)], ids=str)
def test_the_table_of_a_rotation(rot, kw):
    names = {"low": "low_turns", "high": "high_turns", "trained": "trained_tokens"}
    r = S.rope_plan(rot, layout=S.SIF_ROPE_INTERLEAVED, magnitude=1.25, **{names.get(k, k): HOW[v] if k == "scaling" else v for k, v in kw.items()})
    want = frequencies(rot, **kw) / (2 * math.pi)
    got = torch.tensor(list(r.turns), dtype=torch.float64)
    assert (r.rot_dim, r.layout, r.magnitude) == (rot, S.SIF_ROPE_INTERLEAVED, 1.25)
    # a power, a product and two quotients in 64 bits, the power's exponent up to 13 (log 500000)
    assert torch.all((got[:rot // 2] - want).abs() <= 2.0 ** -46 * want) and not got[rot // 2:].any()


def test_scaled_frequencies_at_their_ends():
    """The base's factor divides the lowest frequency by `factor` and leaves the highest; by parts, fast pairs stay and slow ones are divided."""
    plain, base = (torch.tensor(list(S.rope_plan(64, **kw).turns)[:32], dtype=torch.float64) for kw in (dict(), dict(scaling=S.SIF_ROPE_BASE, factor=8.0)))
    assert base[0] == plain[0] and abs(float(plain[31] / base[31]) - 8.0) < 1e-12
    parts = torch.tensor(list(S.rope_plan(64, scaling=S.SIF_ROPE_PARTS, factor=8.0, trained_tokens=4096).turns)[:32], dtype=torch.float64)
    ratio = plain / parts
    assert ratio[0] == 1.0 and abs(float(ratio[31]) - 8.0) < 1e-12 and torch.all(ratio[1:] >= ratio[:-1])


def test_turning_back():
    x = torch.randn(9, 3, 80, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
    pos, f = torch.tensor([0, 1, 5, -7, 1000, 12345678, 2 ** 31 - 1, 3, 4]), frequencies(48)
    for inter in (False, True):
        y, _ = turned(x, pos, f, inter)
        z, _ = turned(y, pos, f, inter, back=True)
        assert torch.allclose(z, x, atol=1e-13, rtol=0) and torch.equal(y[0], x[0]) and torch.equal(y[..., 48:], x[..., 48:])
        assert torch.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    # a pair turns by its angle: (1, 0) becomes (cos, sin)
    e = torch.zeros(1, 1, 16, dtype=torch.float64)
    e[..., 2] = 1
    y, _ = turned(e, torch.tensor([3]), frequencies(16), False)
    a = 3 * 10000 ** -0.25
    assert abs(float(y[0, 0, 2]) - math.cos(a)) < 1e-15 and abs(float(y[0, 0, 10]) - math.sin(a)) < 1e-15


def test_4_bits_are_at_most_half_a_step_off():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(400, 64, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-40, 40, (400, 1), generator=g).double())
    code, byte = to_e2m1(x)
    y = from_e2m1(code, byte)
    p = torch.exp2(byte.double() - 127).repeat_interleave(32, -1)
    a = (y / p).abs()
    step = torch.where(a >= 4, 2.0, torch.where(a >= 2, 1.0, 0.5))
    assert torch.all((x - y).abs() <= p * step / 2) and torch.all(x.abs() <= 7 * p)
    assert torch.all(x.unflatten(-1, (-1, 32)).abs().amax(-1) > 3.5 * torch.exp2(byte.double() - 127))      # no smaller power would do
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0, -0.25, -5.0, -0.0] + [0.0] * 20, dtype=torch.float64)
    assert (from_e2m1(*to_e2m1(ties))[:12]).tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -4, 0]
    odd = torch.zeros(4, 32, dtype=torch.float64)
    odd[0, 3], odd[1, 4], odd[2, 0], odd[3, 0] = math.nan, -math.inf, 2.0 ** -140, 6 * 2.0 ** -127
    code, byte = to_e2m1(odd)
    assert byte[:, 0].tolist() == [255, 253, 0, 0] and code[1, 4] == 15 and code[2].sum() == 0 and code[3, 0] == 7


def test_the_layout_in_4_bits():
    r = Rows("e2m1", [5], 16, kv_heads=1, d=64, layers=1, spare=0)
    k, v = r.raw("k")[0, 0, 0], r.raw("v")[0, 0, 0]
    assert k.numel() == v.numel() == 16 * 64 * 17 // 32
    for tok, d in ((0, 0), (3, 17), (15, 63), (7, 32)):
        assert k[tok * 32 + d // 2] >> (4 * (d % 2)) & 15 == r.code["k"][0, 0, 0, tok, d]
        assert v[(d // 32 * 16 + d % 16) * 16 + tok] >> (4 * (d % 32 // 16)) & 15 == r.code["v"][0, 0, 0, tok, d]
        assert k[16 * 32 + d // 32 * 16 + tok] == r.power["k"][0, 0, 0, tok, d // 32] and v[16 * 32 + tok * 2 + d // 32] == r.power["v"][0, 0, 0, tok, d // 32]


def test_the_reference_of_sampling():
    x = [1.0, 3.0, 2.0, 3.0, -math.inf, math.nan]
    assert sample(x, 0.0, 0.0) == (1, 0.0, 1)
    assert sample(x, 0.99, top_k=1) == (1, 0.0, 1) and sample(x, 0.99, top_k=2)[0] == 3 and sample(x, 0.0, top_k=3)[2] == 3
    assert sample(x, 0.99)[0] == 3 and sample(x, 0.0)[0] == 0 and sample(x, 0.0)[2] == 4
    assert sample(x, 0.5, top_p=0.0)[2] == 1 and sample(x, 0.5, min_p=1.0)[2] == 2 and sample([-math.inf], 0.5) == (-1, -math.inf, 0)
    assert sample([0.0] * 10, 0.35) == (3, pytest.approx(math.log(0.1)), 10) and sample([0.0] * 10, 0.35, top_p=0.5)[2] == 5
