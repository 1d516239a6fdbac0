"""The serving operators' C entry points and binding on the host: structures, workspace, and what they
refuse before any device work (no GPU needed)."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import _lib, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E_ARG, E_SHAPE, E_DTYPE, E_WORKSPACE, E_UNSUPPORTED = -1, -2, -3, -4, -6
P = C.c_void_p(1 << 20)        # a well-aligned address that nothing may read
ODD = C.c_void_p((1 << 20) + 8)


def fields(struct):
    """(name, count) of a structure's members in the header, in order."""
    text = open(os.path.join(ROOT, "include", "ftcnn.h")).read()
    body = re.search(r"typedef struct \{((?:(?!typedef).)*?)\} %s;" % struct, text, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    res = []
    for line in body.split(";"):
        names = re.sub(r"^\s*(int32_t|int64_t|float|double)\s", "", line)
        for name in names.split(","):
            m = re.match(r"\s*(\w+)(?:\[(\d+)\])?\s*$", name)
            if m:
                res.append((m.group(1), int(m.group(2) or 1)))
    return res


@pytest.mark.parametrize("name,ctype,packed", [
    ("ftcnn_rope_scaling", _lib.RopeScaling, None), ("ftcnn_rope_desc", _lib.RopeDesc, paged._ROPE),
    ("ftcnn_append_desc", _lib.AppendDesc, paged._APPEND), ("ftcnn_attention_desc", _lib.AttentionDesc, paged._ATTENTION)])
def test_structures_match_the_header(name, ctype, packed):
    ours = [(f, getattr(t, "_length_", 1)) for f, t in ctype._fields_]
    assert ours == fields(name)
    if packed is not None:
        assert packed.size == C.sizeof(ctype)


def rope(**kw):
    d = _lib.RopeDesc(0, 4, 8, 2, 64, 64, 0, 100, 0, 1e-6)
    for s in (d.q_stride, d.k_stride, d.q_out_stride, d.k_out_stride):
        s[0], s[1] = 512, 64
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def append(**kw):
    d = _lib.AppendDesc(0, 4, 2, 64, 64, 0, 100, 0, 10, 16, 1e-6)
    d.k_stride[0] = d.v_stride[0] = 128
    for s in (d.k_cache_stride, d.v_cache_stride):
        s[0], s[1], s[2] = 2048, 64, 1024
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attention(**kw):
    d = _lib.AttentionDesc(1, 2, 2, 8, 2, 64, 10, 16, 5, 1, 0, 1, 80, 0.125)
    for s in (d.q_stride, d.out_stride):
        s[0], s[1] = 512, 64
    for s in (d.k_cache_stride, d.v_cache_stride):
        s[0], s[1], s[2] = 2048, 64, 1024
    d.list_stride = 5
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def call_rope(d, q=P, k=P, pos=P, table=P, qw=P, kw=P, qo=P, ko=P):
    return _lib.load().ftcnn_qk_norm_rope(bytes(d), q, k, pos, table, qw, kw, qo, ko, None)


def call_append(d, k=P, v=P, pos=P, table=P, w=P, slots=P, kc=P, vc=P):
    return _lib.load().ftcnn_kv_append(bytes(d), k, v, pos, table, w, slots, kc, vc, None)


def call_attention(d, q=P, kc=P, vc=P, lists=P, lens=P, starts=P, out=P, lse=P, ws=P):
    return _lib.load().ftcnn_paged_attention(bytes(d), q, kc, vc, lists, lens, starts, out, lse, ws, None)


@pytest.mark.parametrize("kw,code", [
    (dict(max_pos=0), E_SHAPE), (dict(rot=3), E_SHAPE), (dict(rot=0), E_SHAPE), (dict(rot=258), E_SHAPE),
    (dict(scaling=4), E_ARG), (dict(scaling=-1), E_ARG), (dict(base=0.0), E_ARG), (dict(base=float("nan")), E_ARG),
    (dict(amplitude=float("inf")), E_ARG), (dict(scaling=1, factor=0.0), E_ARG),
    (dict(scaling=2, factor=float("nan")), E_ARG), (dict(scaling=3, factor=2.0, original=0, high=32.0, low=1.0), E_ARG),
    (dict(scaling=3, factor=2.0, original=64, high=1.0, low=1.0), E_ARG)])
def test_rope_table_refuses(kw, code):
    sc = _lib.RopeScaling(100, 64, 0, 0, 10000.0, 1.0, 1.0, 32.0, 1.0)
    for k, v in kw.items():
        setattr(sc, k, v)
    assert _lib.load().ftcnn_rope_table(C.byref(sc), P, None) == code
    assert "rope_table" in ft.last_error()


def test_rope_table_refuses_null():
    sc = _lib.RopeScaling(100, 64, 0, 0, 10000.0, 1.0, 1.0, 32.0, 1.0)
    assert _lib.load().ftcnn_rope_table(None, P, None) == E_ARG
    assert _lib.load().ftcnn_rope_table(C.byref(sc), None, None) == E_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), E_DTYPE), (dict(tokens=-1), E_SHAPE), (dict(heads=-1), E_SHAPE), (dict(heads=0, kv_heads=0), E_SHAPE),
    (dict(heads=2**31 - 1, kv_heads=2**31 - 1), E_SHAPE), (dict(tokens=2**31 - 1), E_SHAPE), (dict(dim=0), E_SHAPE),
    (dict(dim=63), E_SHAPE), (dict(dim=258), E_SHAPE), (dict(rot=66), E_SHAPE), (dict(rot=3), E_SHAPE),
    (dict(rot=0), E_SHAPE), (dict(layout=2), E_ARG), (dict(max_pos=0), E_SHAPE), (dict(eps=-1.0), E_ARG),
    (dict(eps=float("nan")), E_ARG), (dict(eps=float("inf")), E_ARG), (dict(weight_dtype=1), E_DTYPE)])
def test_qk_norm_rope_refuses(kw, code):
    assert call_rope(rope(**kw)) == code
    assert "qk_norm_rope" in ft.last_error()


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(pos=None), dict(table=None)])
def test_qk_norm_rope_refuses_missing_pointers(kw):
    assert call_rope(rope(), **kw) == E_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), E_DTYPE), (dict(tokens=-1), E_SHAPE), (dict(kv_heads=0), E_SHAPE), (dict(dim=2048), E_SHAPE),
    (dict(pages=0), E_SHAPE), (dict(page=0), E_SHAPE), (dict(rot=128), E_SHAPE), (dict(layout=-1), E_ARG),
    (dict(max_pos=-5), E_SHAPE), (dict(eps=float("nan")), E_ARG), (dict(weight_dtype=7), E_DTYPE)])
def test_kv_append_refuses(kw, code):
    assert call_append(append(**kw)) == code
    assert "kv_append" in ft.last_error()


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(pos=None), dict(table=None), dict(slots=None),
                                dict(kc=None), dict(vc=None)])
def test_kv_append_refuses_missing_pointers(kw):
    assert call_append(append(), **kw) == E_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), E_DTYPE), (dict(batch=-1), E_SHAPE), (dict(tokens=-1), E_SHAPE), (dict(heads=0), E_SHAPE),
    (dict(kv_heads=0), E_SHAPE), (dict(heads=7), E_SHAPE), (dict(pages=0), E_SHAPE), (dict(page=0), E_SHAPE),
    (dict(list_len=-1), E_SHAPE), (dict(max_q=-1), E_SHAPE), (dict(max_kv=-1), E_SHAPE), (dict(dim=0), E_UNSUPPORTED),
    (dict(dim=60), E_UNSUPPORTED), (dict(dim=264), E_UNSUPPORTED), (dict(tokens=2**31 - 1), E_SHAPE),
    (dict(list_len=2**30, page=64), E_SHAPE), (dict(window=-1), E_ARG), (dict(window=4, causal=0), E_ARG),
    (dict(scale=0.0), E_ARG), (dict(scale=-1.0), E_ARG), (dict(scale=float("nan")), E_ARG),
    (dict(scale=float("inf")), E_ARG)])
def test_paged_attention_refuses(kw, code):
    d = attention(**kw)
    assert call_attention(d) == code
    assert "paged_attention" in ft.last_error()
    assert _lib.load().ftcnn_paged_attention_workspace_bytes(bytes(d)) == 0


@pytest.mark.parametrize("kw", [dict(q=None), dict(kc=None), dict(vc=None), dict(lists=None), dict(lens=None),
                                dict(out=None)])
def test_paged_attention_refuses_missing_pointers(kw):
    assert call_attention(attention(), **kw) == E_ARG


@pytest.mark.parametrize("kw", [dict(q=ODD), dict(kc=ODD), dict(vc=ODD), dict(out=ODD)])
def test_paged_attention_refuses_rows_off_16_bytes(kw):
    assert call_attention(attention(), **kw) == E_UNSUPPORTED


@pytest.mark.parametrize("field,i,value", [
    ("q_stride", 1, 60), ("out_stride", 0, 513), ("k_cache_stride", 1, 68), ("v_cache_stride", 2, 1028),
    ("k_cache_stride", 0, -2048), ("v_cache_stride", 0, (1 << 29) + 8)])
def test_paged_attention_refuses_strides(field, i, value):
    d = attention()
    getattr(d, field)[i] = value
    assert call_attention(d) == E_UNSUPPORTED


def test_paged_attention_refuses_tokens_without_an_owner():
    assert call_attention(attention(tokens=3), starts=None) == E_SHAPE


def test_paged_attention_workspace():
    """A few rows over many keys are split, and need room; short ones are not."""
    L = _lib.load()
    few, long = attention(list_len=4, max_kv=64), attention(list_len=8192, max_kv=100000)
    assert L.ftcnn_paged_attention_workspace_bytes(bytes(few)) == 0
    need = L.ftcnn_paged_attention_workspace_bytes(bytes(long))
    assert need > 0 and need % 256 == 0
    assert call_attention(long, ws=None) == E_WORKSPACE
    assert call_attention(long, ws=C.c_void_p((1 << 20) + 16)) == E_WORKSPACE
    assert L.ftcnn_paged_attention_workspace_bytes(None) == 0
    # what the plan takes stays within what fits on the device at a time, whatever the sizes
    for kw in (dict(list_len=2**26, max_kv=0), dict(batch=4096, tokens=4096, list_len=8192, max_kv=0),
               dict(batch=1, tokens=1 << 20, max_q=0, list_len=2**26, max_kv=0)):
        assert L.ftcnn_paged_attention_workspace_bytes(bytes(attention(**kw))) < 1 << 30


def test_nothing_to_do_is_no_launch():
    assert call_rope(rope(tokens=0), q=None, k=None, qo=None, ko=None) == 0
    assert call_append(append(tokens=0), k=None, v=None, slots=None, kc=None, vc=None) == 0
    assert call_attention(attention(tokens=0, batch=0), q=None, out=None) == 0


def test_null_descriptors():
    L = _lib.load()
    assert L.ftcnn_qk_norm_rope(None, *[P] * 8, None) == E_ARG
    assert L.ftcnn_kv_append(None, *[P] * 8, None) == E_ARG
    assert L.ftcnn_paged_attention(None, *[P] * 9, None) == E_ARG


def test_binding_refuses_host_tensors_and_names():
    q, c = torch.zeros(2, 4, 64), torch.zeros(3, 16, 2, 64)
    i32 = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ft.FtcnnError, match="on a device"):
        paged.qk_norm_rope(q, None)
    with pytest.raises(ft.FtcnnError, match="neither"):
        paged.qk_norm_rope(None, None)
    with pytest.raises(ft.FtcnnError, match="on a device"):
        paged.kv_append(q[:, :2], q[:, :2], c, c, i32.long())
    with pytest.raises(ft.FtcnnError, match="on a device"):
        paged.paged_attention(q, c, c, i32.view(2, 1), i32)
    with pytest.raises(ft.FtcnnError, match="scaling"):
        paged.rope_table(10, 4, scaling="other")
    with pytest.raises(ft.FtcnnError, match="rot"):
        paged.rope_table(10, 5)


def test_cache_rows_of_tokens():
    cache = paged.PagedCache(6, 4, 2, 8, "f32", device="cpu")
    assert cache.k.shape == (6, 4, 2, 8) and cache.k.stride() == (64, 8, 32, 1)
    lists = torch.tensor([[5, 1, 0], [2, 3, 4]], dtype=torch.int32)
    seq, pos = torch.tensor([0, 0, 1, 1], dtype=torch.int32), torch.tensor([3, 4, 0, 11], dtype=torch.int32)
    assert cache.slots(lists, seq, pos).tolist() == [23, 4, 8, 19]
