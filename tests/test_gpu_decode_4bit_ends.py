"""Attention over a cache in 4 bits where numbers end: held keys past the largest in bf16."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from rows_reference import Rows
from test_gpu_decode_4bit import _attend, _q

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV

MOST = 3.3895313892515355e38          # the largest number in bf16: held as 4 * 2^126, an infinity as 6 * 2^126


def _put(rows, x, s, t, d, **elements):
    """Token t of sequence s becomes zeros and the given elements, in all heads."""
    y = torch.zeros(rows.h, rows.d, dtype=torch.float64)
    for at, value in elements.items():
        y[:, int(at[1:])] = value
    rows.put(x, 0, s, t, y)


@pytest.mark.parametrize("d", [64, 128])
def test_a_query_of_zeros_and_keys_past_the_largest(d):
    """Zero times what is held is zero: every token counts alike but those whose keys the other elements of q see."""
    rows = Rows("e2m1", [40], 16, 1, d, layers=1, seed=5)
    _put(rows, "k", 0, 3, d, e3=math.inf, e40=-MOST)
    _put(rows, "k", 0, 17, d, e19=-math.inf)
    q = _q(5, 1, 3 * d).view(3, d)
    q[0] = 0.0
    q[1, 3], q[1, 19], q[1, 40] = 0.0, 0.0, -0.0
    q[2, :32] = 0.0
    q[2, 40] = 0.0
    _attend(rows, q.reshape(1, -1), 3)


@pytest.mark.parametrize("d", [64, 128])
def test_small_queries_and_keys_past_the_largest(d):
    """Products of about one from keys of 2^125 to 2^129 and queries of 2^-126."""
    g = torch.Generator().manual_seed(d)
    rows = Rows("e2m1", [70, 1, 200], 32, 2, d, layers=1, seed=4)
    rows.power["k"][..., 0] = torch.randint(252, 255, rows.power["k"].shape[:-1], generator=g).to(torch.uint8)
    q = _q(4, 3, 4 * d).view(3, 4, d)
    q[..., :32] = ((1 + torch.rand(3, 4, 32, generator=g)) * torch.randint(0, 2, (3, 4, 32), generator=g).mul(2).sub(1) * 2.0 ** -126).to(torch.bfloat16)
    q[:, 1, :32:3], q[:, 3, 32:] = 0.0, 0.0
    _attend(rows, q.flatten(1), 4)
    _attend(rows, q.flatten(1), 4, scale=0.01)
