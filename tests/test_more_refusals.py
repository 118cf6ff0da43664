"""What rotations, writing with the rotation on the way, reading back, 4-bit caches and the choice of a token refuse: checked on the host before anything is launched, so
without a GPU."""
import ctypes as C
import math

import pytest
import torch

import paper_2503_02550_amd as S
from test_operator_refusals import BAD_CACHE, BAD_LISTS, _cache, _decode, _i32, _refused

AT, OFF = 1 << 20, (1 << 20) + 8


def _set(a, change):
    for name, value in change.items():
        setattr(a, name, value)
    return a


# ---- the table of a rotation ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=8), dict(rot_dim=72), dict(rot_dim=272), dict(layout=2), dict(scaling=4), dict(base=0.5), dict(base=-1.0), dict(base=math.nan),
                                 dict(base=math.inf), dict(magnitude=math.nan), dict(magnitude=math.inf), dict(magnitude=1e39), dict(scaling=S.SIF_ROPE_LINEAR, factor=0.0),
                                 dict(scaling=S.SIF_ROPE_BASE, factor=-2.0), dict(scaling=S.SIF_ROPE_PARTS, factor=math.nan, trained_tokens=100.0), dict(scaling=S.SIF_ROPE_PARTS, factor=2.0),
                                 dict(scaling=S.SIF_ROPE_PARTS, factor=2.0, trained_tokens=100.0, low_turns=4.0, high_turns=4.0),
                                 dict(scaling=S.SIF_ROPE_PARTS, factor=2.0, trained_tokens=100.0, low_turns=math.nan), dict(scaling=S.SIF_ROPE_LINEAR, factor=1e-3)], ids=str)
def test_a_table_is_refused(bad):
    with pytest.raises(S.SifError) as e:
        S.rope_plan(**{**dict(rot_dim=64), **bad})
    assert e.value.status == S.SIF_E_INVAL and "rope_plan" in str(e.value)


def test_a_table_without_its_size_or_place():
    d, r = S.sif_rope_desc(), S.sif_rope()
    d.struct_size, d.rot_dim, d.base, d.magnitude = C.sizeof(d) - 8, 64, 10000.0, 1.0
    assert S.lib.sif_rope_plan(d, r) == S.SIF_E_INVAL and S.lib.sif_rope_plan(None, r) == S.SIF_E_INVAL
    d.struct_size = C.sizeof(d)
    assert S.lib.sif_rope_plan(d, None) == S.SIF_E_INVAL and S.lib.sif_rope_plan(d, r) == S.SIF_OK


BAD_TABLE = [dict(struct_size=1), dict(layout=7), dict(rot_dim=0), dict(rot_dim=40), dict(rot_dim=80), dict(magnitude=math.inf), ("turns", 1.5), ("turns", math.nan), ("turns", -2.0)]


def _table(bad):
    r = S.rope_plan(64)
    if isinstance(bad, tuple):
        r.turns[31] = bad[1]
        return r
    return _set(r, bad)


# ---- turning rows --------------------------------------------------------------------------------------------------
def _rope(**change):
    a = S.sif_rope_args()
    a.struct_size = C.sizeof(a)
    a.rows, a.heads, a.kv_heads, a.d_head, a.seq = 8, 4, 2, 64, 8
    a.ld_q = a.ld_q_out = 256
    a.ld_k = a.ld_k_out = 128
    a.q_dev = a.q_out_dev = a.k_dev = a.k_out_dev = AT
    return _set(a, change)


@pytest.mark.parametrize("change", [dict(struct_size=4), dict(rows=0), dict(rows=1 << 31), dict(heads=0), dict(heads=1 << 15), dict(kv_heads=1 << 15), dict(d_head=0), dict(d_head=60), dict(d_head=32), dict(d_head=264), dict(seq=0),
                                    dict(inverse=2), dict(q_dev=None), dict(q_out_dev=None), dict(k_dev=None), dict(k_out_dev=None), dict(q_dev=OFF), dict(q_out_dev=OFF), dict(k_dev=OFF), dict(k_out_dev=OFF),
                                    dict(positions_dev=AT + 2), dict(ld_q=248), dict(ld_q=260, ld_q_out=260), dict(ld_q_out=264), dict(ld_k=120), dict(ld_k_out=136), dict(ld_q=1 << 27, ld_q_out=1 << 27)], ids=str)
def test_turning_rows_is_refused(change):
    assert S.lib.sif_k_rope(S.rope_plan(64), _rope(**change), None) == S.SIF_E_INVAL and S.last_error().startswith("rope")


@pytest.mark.parametrize("bad", BAD_TABLE, ids=str)
def test_a_bad_table_is_refused(bad):
    assert S.lib.sif_k_rope(_table(bad), _rope(), None) == S.SIF_E_INVAL
    assert S.lib.sif_k_kv_append(_cache(), _table(bad), _append(), None) == S.SIF_E_INVAL
    assert S.lib.sif_k_rope(None, _rope(), None) == S.SIF_E_INVAL and S.lib.sif_k_rope(S.rope_plan(64), None, None) == S.SIF_E_INVAL


# ---- writing and reading rows --------------------------------------------------------------------------------------
def _append(**change):
    a = S.sif_kv_append_args()
    a.struct_size = C.sizeof(a)
    a.layer, a.n, a.rows, a.heads = 1, 2, 2, 4
    a.ld_q = a.ld_q_out = 256
    a.ld_k = a.ld_v = 128
    a.k_dev = a.v_dev = a.q_dev = a.q_out_dev = AT
    return _set(a, change)


BAD_ROWS = [dict(layer=2), dict(k_dev=None), dict(v_dev=None), dict(k_dev=OFF), dict(v_dev=OFF), dict(ld_k=120), dict(ld_v=129), dict(n=0, rows=0), dict(rows=0), dict(rows=3), dict(n=(1 << 27) + 1, rows=(1 << 27) + 1),
            dict(seqs_dev=AT + 2), dict(starts_dev=AT + 2)]


@pytest.mark.parametrize("change", BAD_ROWS + [dict(struct_size=8), dict(heads=1025), dict(q_dev=None), dict(q_out_dev=None), dict(q_dev=OFF), dict(q_out_dev=OFF), dict(ld_q=248), dict(ld_q_out=260),
                                               dict(ld_q_out=264), dict(seqs_dev=AT, starts_dev=AT, n=(1 << 14) + 1)], ids=str)
def test_appending_is_refused(change):
    for dtype in (S.SIF_BF16, S.SIF_E4M3, S.SIF_E2M1):
        assert S.lib.sif_k_kv_append(_cache(dtype=dtype), S.rope_plan(64), _append(**change), None) == S.SIF_E_INVAL and S.last_error().startswith("kv_append")
    assert S.lib.sif_k_kv_append(_cache(), S.rope_plan(64), None, None) == S.SIF_E_INVAL


@pytest.mark.parametrize("change", BAD_ROWS, ids=str)
def test_reading_and_4_bit_writing_are_refused(change):
    x = {**dict(layer=1, k_dev=AT, v_dev=AT, ld_k=128, ld_v=128, seqs_dev=None, starts_dev=None, n=2, rows=2), **change}
    rows = (x["layer"], x["k_dev"], x["v_dev"], x["ld_k"], x["ld_v"], x["seqs_dev"], x["starts_dev"], x["n"], x["rows"], None)
    for dtype in (S.SIF_BF16, S.SIF_E4M3, S.SIF_E2M1):
        assert S.lib.sif_k_kv_read(C.byref(_cache(dtype=dtype)), *rows) == S.SIF_E_INVAL and S.last_error().startswith("kv_read")
    assert S.lib.sif_k_kv_write(C.byref(_cache(dtype=S.SIF_E2M1)), *rows) == S.SIF_E_INVAL


@pytest.mark.parametrize("change", BAD_CACHE, ids=str)
def test_rows_of_a_bad_cache(change):
    c = _cache(**change)
    assert S.lib.sif_k_kv_append(c, S.rope_plan(64), _append(), None) == S.SIF_E_INVAL
    assert S.lib.sif_k_kv_read(c, 0, AT, AT, 128, 128, None, None, 2, 2, None) == S.SIF_E_INVAL
    assert S.lib.sif_k_kv_append(None, S.rope_plan(64), _append(), None) == S.lib.sif_k_kv_read(None, 0, AT, AT, 128, 128, None, None, 2, 2, None) == S.SIF_E_INVAL


def test_a_4_bit_cache():
    """It has no scales beside its pages; all that a bad cache is refused for holds for it too."""
    assert S.sif_kv_workspace_bytes(_cache(dtype=S.SIF_E2M1)) == S.sif_kv_workspace_bytes(_cache())
    for bad in (dict(k_scale_dev=AT), dict(v_scale_dev=AT), dict(d_head=96), dict(page_tokens=8), dict(k_dev=OFF)):
        with pytest.raises(S.SifError):
            S.sif_kv_workspace_bytes(_cache(dtype=S.SIF_E2M1, **bad))
    with pytest.raises(S.SifError):
        S.sif_kv_workspace_bytes(_cache(dtype=4))
    for bad in (dict(layer=2), dict(heads=3), dict(ld_q=248), dict(q_dev=8), dict(scale=-1.0)):
        assert S.lib.sif_k_attn_decode(_cache(dtype=S.SIF_E2M1), _decode(**bad), None) == S.SIF_E_INVAL
    long = _cache(dtype=S.SIF_E2M1, table_ld=100000)
    need = S.sif_attn_decode_workspace_bytes(long, _decode())
    assert need > 256 and S.lib.sif_k_attn_decode(long, _decode(workspace_bytes=need - 1), None) == S.SIF_E_NOMEM


def test_the_binding_of_a_4_bit_cache():
    k = torch.zeros(1, 3, 2, 16 * 64 * 17 // 32, dtype=torch.uint8)
    x = dict(k=k, v=k.clone(), table=torch.zeros(2, 2, dtype=torch.int32), lengths=torch.zeros(2, dtype=torch.int32), refs=torch.zeros(3, dtype=torch.int32), dtype=S.SIF_E2M1, page_tokens=16)
    c = S.kv_cache(**x)
    assert (c.layers, c.n_pages, c.kv_heads, c.d_head, c.dtype) == (1, 3, 2, 64, S.SIF_E2M1)
    wide = torch.zeros(1, 3, 2, 32 * 128 * 17 // 32, dtype=torch.uint8)
    assert S.kv_cache(**{**x, "k": wide, "v": wide, "page_tokens": 32}).d_head == 128
    for bad in (dict(k=k.to(torch.int8)), dict(k=k[..., :-1]), dict(k=k[..., :-16].contiguous(), v=k[..., :-16].contiguous()), dict(v=wide), dict(k=k.float(), v=k.float()), dict(page_tokens=0),
                dict(k=k[:, :2], v=k[:, :2])):
        with pytest.raises(S.SifError):
            S.kv_cache(**{**x, **bad})


# ---- a token for every row -----------------------------------------------------------------------------------------
def _sample(**change):
    a = S.sif_sample_args()
    a.struct_size = C.sizeof(a)
    a.dtype, a.n, a.vocab, a.ld, a.temperature, a.top_p = S.SIF_F32, 2, 100, 104, 1.0, 1.0
    a.logits_dev = a.random_dev = a.token_dev = AT
    return _set(a, change)


@pytest.mark.parametrize("change", [dict(struct_size=0), dict(dtype=S.SIF_E4M3), dict(dtype=7), dict(n=0), dict(n=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 18) + 1, ld=(1 << 18) + 8), dict(ld=96), dict(ld=108),
                                    dict(temperature=-1.0), dict(temperature=math.nan), dict(logits_dev=None), dict(token_dev=None), dict(random_dev=None), dict(random_dev=None, temperature=0.0, temperature_dev=AT),
                                    dict(logits_dev=OFF), dict(token_dev=AT + 1), dict(random_dev=AT + 2), dict(logprob_dev=AT + 3), dict(kept_dev=AT + 2), dict(temperature_dev=AT + 1), dict(top_k_dev=AT + 2),
                                    dict(top_p_dev=AT + 2), dict(min_p_dev=AT + 1)], ids=str)
def test_choosing_a_token_is_refused(change):
    assert S.lib.sif_k_sample(_sample(**change), None) == S.SIF_E_INVAL and S.last_error().startswith("sample")
    assert S.lib.sif_k_sample(None, None) == S.SIF_E_INVAL


# ---- tensors -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bad", BAD_LISTS, ids=["int64", "float", "short", "strided"])
def test_the_binding_refuses_lists(bad):
    z, f = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4)
    good = _i32(0, 1, 2, 3, 4)
    for call in (lambda: S.rope_args(z, z, 4, 2, 64, positions=bad), lambda: S.kv_append_args(z, z, 4, seqs=bad), lambda: S.kv_append_args(z, z, 3, rows=4, starts=bad),
                 lambda: S.sif_k_kv_read(_cache(), 0, z, z, bad, 4), lambda: S.sif_k_kv_read(_cache(), 0, z, z, None, 3, starts=bad, rows=4),
                 lambda: S.sample_args(z, bad, 4, 128, random=f), lambda: S.sample_args(z, good, 4, 128, random=f, top_k=bad), lambda: S.sample_args(z, good, 4, 128, random=f, kept=bad)):
        assert "int32" in _refused(call)


def test_the_binding_refuses_rows_and_numbers():
    z, f, good = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4), _i32(0, 1, 2, 3)
    turned = torch.zeros(128, 4, dtype=torch.bfloat16).t()
    for bad in (z.float(), z.half(), turned):
        for name in ("q", "q_out", "k", "k_out"):
            _refused(lambda: S.rope_args(**{**dict(q=z, q_out=z, k=z, k_out=z, rows=4, heads=2, kv_heads=2, d_head=64, seq=4), name: bad}))
        for name in ("k", "v", "q", "q_out"):
            _refused(lambda: S.kv_append_args(**{**dict(k=z, v=z, q=z, q_out=z, n=4, heads=2), name: bad}))
        _refused(lambda: S.sif_k_kv_read(_cache(), 0, bad, z, None, 4))
        _refused(lambda: S.sif_k_kv_read(_cache(), 0, z, bad, None, 4))
    for bad in (z.half(), z.double(), turned, 5):
        _refused(lambda: S.sample_args(bad, good, 4, 128, random=f))
    for bad in (f.double(), torch.zeros(8)[::2], f[:3], good):
        for name in ("random", "temperature", "top_p", "min_p", "logprob"):
            _refused(lambda: S.sample_args(**{**dict(logits=z, token=good, n=4, vocab=128, random=f), name: bad}))
    a = S.sample_args(z.float(), good, 4, 128, random=f, temperature=f, top_k=3, top_p=0.5)
    assert (a.dtype, a.ld, a.top_k, a.top_p, a.temperature_dev) == (S.SIF_F32, 128, 3, 0.5, f.data_ptr())


def test_the_binding_refuses_rows_that_are_not_there():
    """A tensor that ends in front of the last row that a call would read or write."""
    z, f, good = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(5), _i32(0, 1, 2, 3, 4)
    wide = torch.zeros(4, 256, dtype=torch.bfloat16)
    for name in ("q", "q_out", "k", "k_out"):
        x = {**dict.fromkeys(("q", "q_out", "k", "k_out"), wide), "heads": 4, "kv_heads": 4, "d_head": 64, "seq": 4}
        S.rope_args(**x, rows=4)
        S.rope_args(**{**x, name: wide[:, :128], "heads": 2, "kv_heads": 2}, rows=4)
        S.rope_args(**{**x, name: wide.view(4, 4, 64)}, rows=4)
        for bad in (wide[:3], wide.view(-1)[:-1], wide.view(4, 4, 64)[:3], wide[:, :128], wide[:0], wide[0]):
            assert f"{name} must hold 4 rows of 256" in _refused(lambda: S.rope_args(**{**x, name: bad}, rows=4))
        _refused(lambda: S.rope_args(**x, rows=5))
    for name in ("k", "v", "q", "q_out"):
        x = {**dict.fromkeys(("k", "v", "q", "q_out"), z), "heads": 2}
        S.kv_append_args(**x, n=4)
        S.kv_append_args(**x, n=2, rows=4)
        for bad in (z[:3], z[:0], z.view(-1)[:384].view(3, 128)):
            assert f"{name} must hold 4 rows" in _refused(lambda: S.kv_append_args(**{**x, name: bad}, n=2, rows=4))
        _refused(lambda: S.kv_append_args(**x, n=5))
    for bad in (z[:3], z.view(-1)[:-1], z[:, :64], z[:0]):
        assert "k must hold 4 rows of 128" in _refused(lambda: S.sif_k_kv_read(_cache(), 0, bad, z, None, 4))
        assert "v must hold 4 rows of 128" in _refused(lambda: S.sif_k_kv_read(_cache(), 0, z, bad, None, 2, starts=_i32(0, 1, 4), rows=4))
    for x in (z, z.float()):
        S.sample_args(x, good, 4, 121, random=f)
        S.sample_args(x[:, :100], good, 4, 100, random=f)
        for bad in (x[:3], x.view(-1)[:511], x[:, :100], x[:0], x[0]):
            assert "logits must hold 4 rows of 128" in _refused(lambda: S.sample_args(bad, good, 4, 128, random=f))
        _refused(lambda: S.sample_args(x, good, 5, 128, random=f))
        _refused(lambda: S.sample_args(x, good, 4, 129, random=f))
        _refused(lambda: S.sample_args(x, good, 3, 128, random=f, ld=256))
