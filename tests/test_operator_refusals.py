"""What the attention operators and the cache's page operations refuse: checked on the host before anything is launched, so without a GPU."""
import ctypes as C
import math

import pytest
import torch

import paper_2503_02550_amd as S


def _window(**change):
    z = torch.zeros(64, 256, dtype=torch.bfloat16)
    f = torch.zeros(64 * 4)
    a = S.window_attn_args(z, z, z, z, heads=4, kv_heads=2, d_head=64, batch=1, seq_q=64, seq_k=64, window=8, sinks=2, lse=f, d_o=z, dq=z, dk=z, dv=z)
    S.set_workspace(a, 1 << 20, 1 << 20)
    a.keep = (z, f)
    for name, value in change.items():
        setattr(a, name, value)
    return a


BAD_WINDOW = [dict(struct_size=8), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(d_head=32), dict(d_head=96), dict(d_head=256), dict(batch=0), dict(seq_q=0),
              dict(seq_k=0), dict(seq_q=(1 << 20) + 1), dict(batch=1 << 21), dict(sinks=129), dict(window=(1 << 30) + 1), dict(scale=-1.0), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(heads=2048, kv_heads=2), dict(q_dev=None), dict(k_dev=None), dict(v_dev=None), dict(o_dev=None), dict(ld_q=248), dict(ld_k=120),
              dict(ld_v=129), dict(ld_o=260), dict(ld_k=1 << 27), dict(q_dev=8), dict(o_dev=4), dict(lse_dev=2), dict(starts_dev=64, rows=0), dict(starts_dev=64, rows=64, seq_q=32),
              dict(starts_dev=66, rows=64)]
BAD_BACKWARD = [dict(lse_dev=None), dict(do_dev=None), dict(dq_dev=None), dict(dk_dev=None), dict(dv_dev=None), dict(ld_do=8), dict(ld_dq=252), dict(ld_dk=120), dict(ld_dv=124),
                dict(do_dev=8), dict(dv_dev=8), dict(workspace_dev=None), dict(workspace_dev=(1 << 20) + 16)]


@pytest.mark.parametrize("change", BAD_WINDOW, ids=str)
def test_window_attention_refuses(change):
    for call in (S.sif_k_window_attn_fwd, S.sif_k_window_attn_bwd):
        with pytest.raises(S.SifError) as e:
            call(_window(**change))
        assert e.value.status == S.SIF_E_INVAL and "window_attn" in str(e.value)


@pytest.mark.parametrize("change", BAD_BACKWARD, ids=str)
def test_window_attention_backward_refuses(change):
    with pytest.raises(S.SifError) as e:
        S.sif_k_window_attn_bwd(_window(**change))
    assert e.value.status == S.SIF_E_INVAL


def test_window_attention_needs_its_whole_workspace():
    n = S.sif_window_attn_bwd_workspace_bytes(_window())
    assert n >= 4 * 64 * 4
    with pytest.raises(S.SifError) as e:
        S.sif_k_window_attn_bwd(_window(workspace_bytes=n - 1))
    assert e.value.status == S.SIF_E_NOMEM
    with pytest.raises(S.SifError):
        S.sif_window_attn_bwd_workspace_bytes(_window(d_head=80))
    for call in (S.lib.sif_k_window_attn_fwd, S.lib.sif_k_window_attn_bwd):
        assert call(None, None) == S.SIF_E_INVAL
    assert S.lib.sif_window_attn_bwd_workspace_bytes(None) == 0


def _cache(**change):
    c = S.sif_kv_cache()
    c.struct_size = C.sizeof(S.sif_kv_cache)
    c.dtype, c.layers, c.kv_heads, c.d_head, c.page_tokens, c.n_pages, c.n_seqs, c.table_ld = S.SIF_BF16, 2, 2, 64, 16, 10, 4, 5
    c.k_dev = c.v_dev = c.table_dev = c.lengths_dev = c.refs_dev = 1 << 20
    for name, value in change.items():
        setattr(c, name, value)
    return c


BAD_CACHE = [dict(struct_size=1), dict(dtype=S.SIF_F32), dict(dtype=7), dict(layers=0), dict(kv_heads=0), dict(d_head=96), dict(d_head=0), dict(page_tokens=0), dict(page_tokens=8),
             dict(page_tokens=48), dict(page_tokens=512), dict(n_pages=0), dict(n_seqs=0), dict(table_ld=0), dict(k_dev=None), dict(v_dev=None), dict(table_dev=None),
             dict(lengths_dev=None), dict(refs_dev=None), dict(k_dev=8), dict(refs_dev=(1 << 20) + 4), dict(table_dev=2), dict(k_scale_dev=1 << 20), dict(layers=1025),
             dict(kv_heads=1025), dict(table_ld=1 << 27), dict(n_pages=(1 << 21) + 1), dict(n_seqs=0x7FFFFFFF)]


def _calls(c):
    lib, at, big = S.lib, 1 << 20, 1 << 40
    p = C.byref(c) if c is not None else None
    return {"reset": lambda: lib.sif_k_kv_reset(p, None), "extend": lambda: lib.sif_k_kv_extend(p, at, at, 2, None, at, big, None),
            "write": lambda: lib.sif_k_kv_write(p, 0, at, at, 128, 128, at, None, 2, 2, None), "fork": lambda: lib.sif_k_kv_fork(p, at, at, 2, None, None),
            "free": lambda: lib.sif_k_kv_free(p, at, 2, None), "trim": lambda: lib.sif_k_kv_trim(p, at, 2, 4, 0, None),
            "compact": lambda: lib.sif_k_kv_compact(p, at, big, None), "copy": lambda: lib.sif_k_kv_copy_pages(p, at, at, 2, None, None),
            "decode": lambda: lib.sif_k_attn_decode(p, C.byref(_decode()), None)}


def _decode(**change):
    z = torch.zeros(4, 256, dtype=torch.bfloat16)
    a = S.attn_decode_args(z, z, n=4, heads=4)
    a.q_dev = a.o_dev = a.workspace_dev = 1 << 20
    a.workspace_bytes = 1 << 40
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change", BAD_CACHE, ids=str)
def test_every_operation_refuses_a_bad_cache(change):
    for name, call in _calls(_cache(**change)).items():
        assert call() == S.SIF_E_INVAL, name
    with pytest.raises(S.SifError):
        S.sif_kv_workspace_bytes(_cache(**change))


def test_no_cache_at_all():
    for name, call in _calls(None).items():
        assert call() == S.SIF_E_INVAL, name
    assert S.lib.sif_kv_workspace_bytes(None) == 0


def test_page_operations_refuse_bad_lists_and_workspaces():
    c, lib, at, big = _cache(), S.lib, 1 << 20, 1 << 40
    p = C.byref(c)
    for n in (0, 1025):
        assert lib.sif_k_kv_extend(p, at, at, n, None, at, big, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_fork(p, at, at, n, None, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_free(p, at, n, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_trim(p, at, n, 4, 0, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_copy_pages(p, at, at, n, None, None) == S.SIF_E_INVAL
    assert lib.sif_k_kv_trim(p, at, 2, 0, 0, None) == S.SIF_E_INVAL                     # a window of nothing
    for src, dst in ((None, at), (at, None)):
        assert lib.sif_k_kv_fork(p, src, dst, 2, None, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_copy_pages(p, src, dst, 2, None, None) == S.SIF_E_INVAL
    need = S.sif_kv_workspace_bytes(c)
    for work, size, status in ((None, big, S.SIF_E_INVAL), (at + 16, big, S.SIF_E_INVAL), (at, need - 1, S.SIF_E_NOMEM)):
        assert lib.sif_k_kv_extend(p, at, at, 2, None, work, size, None) == status
        assert lib.sif_k_kv_compact(p, work, size, None) == status


def test_page_operations_refuse_misaligned_lists():
    c, lib, at, big = _cache(), S.lib, 1 << 20, 1 << 40
    p, off = C.byref(c), at + 2
    for x, y, status in ((off, at, None), (at, off, None), (at, at, off)):
        assert lib.sif_k_kv_extend(p, x, y, 2, status, at, big, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_fork(p, x, y, 2, status, None) == S.SIF_E_INVAL
        assert lib.sif_k_kv_copy_pages(p, x, y, 2, status, None) == S.SIF_E_INVAL
    assert lib.sif_k_kv_free(p, off, 2, None) == S.SIF_E_INVAL
    assert lib.sif_k_kv_trim(p, off, 2, 4, 0, None) == S.SIF_E_INVAL
    for seqs, starts in ((off, None), (at, off)):
        assert lib.sif_k_kv_write(p, 0, at, at, 128, 128, seqs, starts, 2, 2, None) == S.SIF_E_INVAL


@pytest.mark.parametrize("change", [dict(layer=2), dict(k=None), dict(v=None), dict(k=8), dict(ld_k=120), dict(ld_v=129), dict(n=0, rows=0), dict(rows=0), dict(rows=3), dict(n=(1 << 27) + 1, rows=(1 << 27) + 1)], ids=str)
def test_write_refuses(change):
    x = dict(dict(layer=0, k=1 << 20, v=1 << 20, ld_k=128, ld_v=128, n=2, rows=2), **change)
    assert S.lib.sif_k_kv_write(C.byref(_cache()), x["layer"], x["k"], x["v"], x["ld_k"], x["ld_v"], None, None, x["n"], x["rows"], None) == S.SIF_E_INVAL


def test_write_refuses_a_long_list_of_sequences():
    """Each row looks through the list in front of its own entry, so the list's length is limited; entries 0 .. n-1 without a list are not."""
    most, at = 1 << 14, 1 << 20
    p = C.byref(_cache())
    assert S.lib.sif_k_kv_write(p, 0, at, at, 128, 128, at, None, most + 1, most + 1, None) == S.SIF_E_INVAL and "16384" in S.last_error()
    assert S.lib.sif_k_kv_write(p, 0, at, at, 128, 128, at, at, 1 << 27, 1, None) == S.SIF_E_INVAL


@pytest.mark.parametrize("change", [dict(struct_size=4), dict(layer=2), dict(n=0), dict(heads=0), dict(heads=3), dict(q_dev=None), dict(o_dev=None), dict(q_dev=8), dict(o_dev=2),
                                    dict(lse_dev=2), dict(seqs_dev=1), dict(ld_q=248), dict(ld_o=260), dict(scale=-0.5), dict(scale=float("nan")), dict(n=1 << 21)], ids=str)
def test_decode_refuses(change):
    assert S.lib.sif_k_attn_decode(C.byref(_cache()), C.byref(_decode(**change)), None) == S.SIF_E_INVAL


def test_decode_needs_its_workspace_where_it_splits():
    c, a = _cache(table_ld=100000), _decode()
    need = S.sif_attn_decode_workspace_bytes(c, a)
    assert need > 256
    for work, size, status in ((None, need, S.SIF_E_INVAL), ((1 << 20) + 128, need, S.SIF_E_INVAL), (1 << 20, need - 1, S.SIF_E_NOMEM)):
        assert S.lib.sif_k_attn_decode(C.byref(c), C.byref(_decode(workspace_dev=work, workspace_bytes=size)), None) == status
    assert S.sif_attn_decode_workspace_bytes(c, _decode(max_tokens=64)) <= 256            # short sequences: nothing to split
    with pytest.raises(S.SifError):
        S.sif_attn_decode_workspace_bytes(c, _decode(heads=5))
    assert S.lib.sif_attn_decode_workspace_bytes(C.byref(c), None) == 0


def test_a_workspace_planned_for_shorter_sequences_is_refused():
    """Its size goes by max_tokens, so a call with another asks for its own."""
    c = _cache(table_ld=100000)
    short, long = (S.sif_attn_decode_workspace_bytes(c, _decode(max_tokens=m)) for m in (1000, 100000))
    assert short < long
    assert S.lib.sif_k_attn_decode(C.byref(c), C.byref(_decode(max_tokens=100000, workspace_bytes=short)), None) == S.SIF_E_NOMEM


def test_a_scale_whose_base_2_form_is_infinite_is_refused():
    """Exponentials are taken in base 2: past this a score of zero would become NaN."""
    most = 3.4028235e38 * math.log(2.0)
    for scale, refused in ((1.001 * most, True), (0.999 * most, False)):
        assert (S.lib.sif_window_attn_bwd_workspace_bytes(C.byref(_window(scale=scale))) == 0) == refused
        assert (S.lib.sif_attn_decode_workspace_bytes(C.byref(_cache()), C.byref(_decode(scale=scale))) == 0) == refused
        for call in (lambda: S.lib.sif_k_window_attn_fwd(C.byref(_window(scale=scale, q_dev=None)), None), lambda: S.lib.sif_k_attn_decode(C.byref(_cache()), C.byref(_decode(scale=scale, ld_q=0)), None)):
            assert call() == S.SIF_E_INVAL and ("scale" in S.last_error()) == refused


def test_the_binding_refuses_tensors_that_do_not_fit():
    k, v = torch.zeros(1, 3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 3, 2, 64, 16, dtype=torch.bfloat16)
    table, lengths, refs = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = S.kv_cache(k, v, table, lengths, refs, S.SIF_BF16, 16)
    assert (c.layers, c.n_pages, c.kv_heads, c.d_head, c.n_seqs, c.table_ld) == (1, 3, 2, 64, 2, 2)
    for bad in (dict(v=k), dict(k=k.float()), dict(dtype=S.SIF_E4M3), dict(page_tokens=32), dict(refs=refs[:2]), dict(lengths=lengths.long()), dict(table=table[:1]),
                dict(k_scale=torch.zeros(1, 3))):
        x = dict(dict(k=k, v=v, table=table, lengths=lengths, refs=refs, dtype=S.SIF_BF16, page_tokens=16), **bad)
        with pytest.raises(S.SifError):
            S.kv_cache(**x)


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def _refused(call):
    with pytest.raises(S.SifError) as e:
        call()
    assert e.value.status == S.SIF_E_INVAL
    return str(e.value)


BAD_LISTS = [torch.arange(4), torch.zeros(4), _i32(0), _i32(*range(8))[::2]]      # 64 bits (what torch counts in), not whole, too short, not in a row


@pytest.mark.parametrize("bad", BAD_LISTS, ids=["int64", "float", "short", "strided"])
def test_the_binding_refuses_lists_that_the_kernels_would_read_wrongly(bad):
    """The library takes a list as an address: one of 64-bit numbers would be read as twice as many of 32 bits, a short one past its end."""
    c, good, at, big, x = _cache(), _i32(0, 1, 2, 3, 4), 1 << 20, 1 << 40, torch.zeros(4, 128, dtype=torch.bfloat16)
    for call in (lambda: S.sif_k_kv_extend(c, bad, None, 4, at, big), lambda: S.sif_k_kv_extend(c, None, bad, 4, at, big), lambda: S.sif_k_kv_extend(c, None, None, 4, at, big, status=bad),
                 lambda: S.sif_k_kv_write(c, 0, x, x, bad, 4), lambda: S.sif_k_kv_write(c, 0, x, x, None, 3, starts=bad, rows=4),
                 lambda: S.sif_k_kv_fork(c, bad, good, 4), lambda: S.sif_k_kv_fork(c, good, bad, 4), lambda: S.sif_k_kv_fork(c, good, good, 4, status=bad),
                 lambda: S.sif_k_kv_free(c, bad, 4), lambda: S.sif_k_kv_trim(c, bad, 4, 16, 0),
                 lambda: S.sif_k_kv_copy_pages(c, bad, good, 4), lambda: S.sif_k_kv_copy_pages(c, good, bad, 4), lambda: S.sif_k_kv_copy_pages(c, good, good, 4, status=bad)):
        assert "int32" in _refused(call)
    z = torch.zeros(4, 256, dtype=torch.bfloat16)
    assert "int32" in _refused(lambda: S.attn_decode_args(z, z, 4, 4, seqs=bad))
    assert "int32" in _refused(lambda: S.window_attn_args(z, z, z, z, 4, 4, 64, 3, 4, 4, 0, 0, starts=bad, rows=4))


def test_the_binding_refuses_rows_of_another_type_or_order():
    z, f = torch.zeros(64, 256, dtype=torch.bfloat16), torch.zeros(256)
    turned = torch.zeros(256, 64, dtype=torch.bfloat16).t()
    names = ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")
    S.window_attn_args(**dict.fromkeys(names, z), lse=f, heads=4, kv_heads=4, d_head=64, batch=1, seq_q=64, seq_k=64, window=0, sinks=0)
    for bad in (z.float(), z.half(), turned):
        for name in names:
            x = dict(dict.fromkeys(names, z), **{name: bad})
            _refused(lambda: S.window_attn_args(**x, lse=f, heads=4, kv_heads=4, d_head=64, batch=1, seq_q=64, seq_k=64, window=0, sinks=0))
        _refused(lambda: S.attn_decode_args(bad, z, 64, 4))
        _refused(lambda: S.attn_decode_args(z, bad, 64, 4))
        _refused(lambda: S.sif_k_kv_write(_cache(), 0, bad[:4, :128], z[:4, :128], None, 4))
        _refused(lambda: S.sif_k_kv_write(_cache(), 0, z[:4, :128], bad[:4, :128], None, 4))
    for lse in (f.double(), f.to(torch.bfloat16), torch.zeros(512)[::2]):
        _refused(lambda: S.attn_decode_args(z, z, 64, 4, lse=lse))
        _refused(lambda: S.window_attn_args(z, z, z, z, 4, 4, 64, 1, 64, 64, 0, 0, lse=lse))
