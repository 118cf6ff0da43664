"""Windowed attention backward on tensors past 4 GiB, and decoding over pages that several sequences share."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_reference import assert_within, heads_attention, visible

if torch.cuda.is_available():
    import paper_2503_02550_amd as S
    from gpu_util import DEV
    from test_gpu_paged_cache import _filled, _rows
    from test_gpu_window_attention import _inputs


def test_backward_on_rows_past_32_bits():
    """A leading dimension that takes the last rows of all operands and results beyond 4 GiB."""
    d, s, window, sinks, ld = 64, 300, 50, 2, 8 * 1024 * 1024
    q, k, v, do = _inputs(6, s, s, 1, 1, d)
    wide = torch.zeros(s, ld, dtype=torch.bfloat16, device=DEV)      # 5 GB: q, k, v, do, o, dq, dk, dv side by side, a column of zeros behind each
    at = lambda i: wide[:, 128 * i:128 * i + d]      # noqa: E731
    for i, x in enumerate((q, k, v, do)):
        at(i).copy_(x.to(DEV))
    lse = torch.empty(1, s, device=DEV)
    a = S.window_attn_args(at(0), at(1), at(2), at(4), 1, 1, d, 1, s, s, window, sinks, lse=lse, d_o=at(3), dq=at(5), dk=at(6), dv=at(7))
    assert a.ld_q == a.ld_dv == ld and s * ld * 2 > 1 << 32
    size = S.sif_window_attn_bwd_workspace_bytes(a)
    work = torch.empty(size, dtype=torch.uint8, device=DEV)
    S.set_workspace(a, work, size)
    S.sif_k_window_attn_fwd(a)
    S.sif_k_window_attn_bwd(a)
    torch.cuda.synchronize()
    val, tol = heads_attention(q.double(), k.double(), v.double(), 1, 1, d, visible(s, s, window, sinks), 0.125, do.double(), True)
    for i, name in ((4, "o"), (5, "dq"), (6, "dk"), (7, "dv")):
        assert_within(at(i), val[name], tol[name], name)
    assert_within(lse, val["lse"], tol["lse"], "lse")
    assert not any(wide[:, 128 * i + d:128 * i + 128].any() for i in range(8)) and not wide[::100, 1024:].any()


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_over_shared_pages_in_several_splits(e4m3):
    """Answers forked from one long prompt: their pages are one another's but for the last, and each sequence is cut over blocks."""
    lens, d, heads = [9001, 0, 0, 700], 128, 8
    pool = _filled(61, lens, 16, spare=8, wider=2, kv_heads=2, d=d, layers=1, e4m3=e4m3)
    pool.fork([0, 0], [1, 2])
    pool.extend([1, 2, 3], [1, 1, 1], 3)
    pool.write(0, _rows(62, 3, 2 * d), _rows(63, 3, 2 * d), [1, 2, 3], 3)
    pool.check()
    assert pool.ref.table[1][:562] == pool.ref.table[2][:562] == pool.ref.table[0][:562] and len({pool.ref.table[i][562] for i in range(3)}) == 3
    for window, sinks in ((0, 0), (5000, 4)):
        pool.attend(_rows(64, 5, heads * d), heads, 0, [0, 1, 2, 3, 1], window, sinks)
