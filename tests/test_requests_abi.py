"""The C entry points of adapters, attention mass and eviction on the host: structures, workspaces, and what they
refuse before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import _lib, adapters, paged
from test_paged_abi import E_ARG, E_DTYPE, E_SHAPE, E_UNSUPPORTED, E_WORKSPACE, ODD, P, fields


@pytest.mark.parametrize("name,ctype,packed", [
    ("ftcnn_low_rank_desc", _lib.LowRankDesc, adapters._LOW_RANK), ("ftcnn_mass_desc", _lib.MassDesc, paged._MASS),
    ("ftcnn_evict_desc", _lib.EvictDesc, paged._EVICT)])
def test_structures_match_the_header(name, ctype, packed):
    assert [(f, getattr(t, "_length_", 1)) for f, t in ctype._fields_] == fields(name)
    assert packed.size == C.sizeof(ctype)


def filled(d, kw):
    for k, v in kw.items():
        if isinstance(k, tuple):
            getattr(d, k[0])[k[1]] = v
        else:
            setattr(d, k, v)
    return d


def low_rank(kw={}):
    d = _lib.LowRankDesc(1, 10, 64, 128, 4, 16, 64, 128, 128)
    d.a_stride[0], d.a_stride[1], d.b_stride[0], d.b_stride[1] = 1024, 64, 2048, 16
    return filled(d, kw)


def mass(kw={}):
    d = _lib.MassDesc(1, 2, 2, 8, 2, 64, 10, 16, 5, 1, 0, 1, 80, 0.125)
    d.q_stride[0], d.q_stride[1] = 512, 64
    d.k_cache_stride[0], d.k_cache_stride[1], d.k_cache_stride[2] = 2048, 64, 1024
    d.mass_stride, d.list_stride = 80, 5
    return filled(d, kw)


def evict(kw={}):
    d = _lib.EvictDesc(1, 2, 2, 64, 10, 16, 5, 0, 0, 0)
    for s in (d.k_cache_stride, d.v_cache_stride):
        s[0], s[1], s[2] = 2048, 64, 1024
    d.list_stride, d.mass_stride, d.position_stride, d.mass_out_stride, d.position_out_stride = 5, 80, 80, 80, 80
    return filled(d, kw)


def call_low_rank(d, y=P, x=P, a=P, b=P, ids=P, scales=None, ranks=None, out=P, ws=P):
    return _lib.load().ftcnn_low_rank_add(bytes(d), y, x, a, b, ids, scales, ranks, out, ws, None)


def call_mass(d, q=P, k=P, lists=P, lens=P, starts=P, lse=P, m=P, ws=P):
    return _lib.load().ftcnn_attention_mass(bytes(d), q, k, lists, lens, starts, lse, m, ws, None)


def call_evict(d, k=P, v=P, lists=P, lens=P, keep=P, m=P, pos=P, since=P, lo=P, mo=P, po=P, ws=P):
    return _lib.load().ftcnn_evict(bytes(d), k, v, lists, lens, keep, m, pos, since, lo, mo, po, ws, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), E_DTYPE), (dict(tokens=-1), E_SHAPE), (dict(ch=0), E_SHAPE), (dict(m=0), E_SHAPE), (dict(adapters=0), E_SHAPE),
    (dict(rank=0), E_SHAPE), (dict(rank=-8), E_SHAPE), (dict(ch=60), E_UNSUPPORTED), (dict(m=4), E_UNSUPPORTED),
    (dict(rank=12), E_UNSUPPORTED), (dict(rank=136), E_UNSUPPORTED), (dict(x_stride=68), E_UNSUPPORTED),
    (dict(y_stride=-4), E_UNSUPPORTED), (dict(out_stride=130), E_UNSUPPORTED), ({("a_stride", 0): 1028}, E_UNSUPPORTED),
    ({("b_stride", 1): 20}, E_UNSUPPORTED), (dict(tokens=(1 << 30) + 1), E_SHAPE), (dict(ch=(1 << 31) - 8), E_SHAPE), (dict(m=(1 << 31) - 8), E_SHAPE),
    (dict(tokens=1 << 30, m=1 << 30, out_stride=1 << 30), E_SHAPE)])
def test_low_rank_add_refuses(kw, code):
    d = low_rank(kw)
    assert call_low_rank(d) == code
    assert "low_rank_add" in ft.last_error()
    assert _lib.load().ftcnn_low_rank_workspace_bytes(bytes(d)) == 0


def test_low_rank_add_takes_fp32_sizes_of_four():
    assert _lib.load().ftcnn_low_rank_workspace_bytes(bytes(low_rank(dict(dtype=0, ch=60, m=4, rank=12, tokens=5000)))) > 0


@pytest.mark.parametrize("kw", [dict(y=None), dict(x=None), dict(a=None), dict(b=None), dict(ids=None), dict(out=None)])
def test_low_rank_add_refuses_missing_pointers(kw):
    assert call_low_rank(low_rank(), **kw) == E_ARG


@pytest.mark.parametrize("kw", [dict(y=ODD), dict(x=ODD), dict(a=ODD), dict(b=ODD), dict(out=ODD)])
def test_low_rank_add_refuses_rows_off_16_bytes(kw):
    assert call_low_rank(low_rank(), **kw) == E_UNSUPPORTED


def test_low_rank_add_refuses_outputs_that_overlap():
    assert call_low_rank(low_rank(dict(y_stride=256))) == E_ARG             # in place, other strides
    assert call_low_rank(low_rank(dict(out_stride=120)), out=C.c_void_p(1 << 22)) == E_UNSUPPORTED


def test_low_rank_add_workspace():
    L = _lib.load()
    for tokens in (1, 16, 17, 256, 257, 8192, 1 << 20):
        for rank in (8, 64, 128):
            need = L.ftcnn_low_rank_workspace_bytes(bytes(low_rank(dict(tokens=tokens, rank=rank))))
            assert need == 0 if tokens <= 257 else need % 256 == 0 and need >= tokens * rank * 4
    assert L.ftcnn_low_rank_workspace_bytes(None) == 0 and L.ftcnn_low_rank_workspace_bytes(bytes(low_rank(dict(tokens=0)))) == 0
    assert call_low_rank(low_rank(dict(tokens=5000)), ws=None) == E_WORKSPACE
    assert call_low_rank(low_rank(dict(tokens=5000)), ws=C.c_void_p((1 << 20) + 16)) == E_WORKSPACE


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), E_DTYPE), (dict(batch=-1), E_SHAPE), (dict(tokens=-1), E_SHAPE), (dict(heads=0), E_SHAPE),
    (dict(kv_heads=0), E_SHAPE), (dict(heads=7), E_SHAPE), (dict(pages=0), E_SHAPE), (dict(page=0), E_SHAPE),
    (dict(list_len=-1), E_SHAPE), (dict(max_q=-1), E_SHAPE), (dict(max_kv=-1), E_SHAPE), (dict(dim=0), E_UNSUPPORTED),
    (dict(dim=60), E_UNSUPPORTED), (dict(dim=264), E_UNSUPPORTED), (dict(tokens=2**31 - 1), E_SHAPE),
    (dict(list_len=2**30, page=64), E_SHAPE), (dict(window=-1), E_ARG), (dict(window=4, causal=0), E_ARG),
    (dict(scale=0.0), E_ARG), (dict(scale=-1.0), E_ARG), (dict(scale=float("nan")), E_ARG), (dict(scale=3e38), E_ARG)])
def test_attention_mass_refuses(kw, code):
    d = mass(kw)
    assert call_mass(d) == code
    assert "attention_mass" in ft.last_error()
    assert _lib.load().ftcnn_attention_mass_workspace_bytes(bytes(d)) == 0


@pytest.mark.parametrize("kw", [{("q_stride", 1): 60}, {("k_cache_stride", 1): 68}, {("k_cache_stride", 0): -2048},
                                {("k_cache_stride", 2): (1 << 29) + 8}, dict(mass_stride=79), dict(mass_stride=0)])
def test_attention_mass_refuses_strides(kw):
    assert call_mass(mass(kw)) == E_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(lists=None), dict(lens=None), dict(lse=None), dict(m=None)])
def test_attention_mass_refuses_missing_pointers(kw):
    assert call_mass(mass(), **kw) == E_ARG


def test_attention_mass_refuses_what_does_not_fit():
    assert call_mass(mass(), q=ODD) == E_UNSUPPORTED and call_mass(mass(), k=ODD) == E_UNSUPPORTED
    assert call_mass(mass(dict(tokens=3)), starts=None) == E_SHAPE
    wide = mass(dict(tokens=200, max_q=100, list_len=60, max_kv=900, mass_stride=960))
    need = _lib.load().ftcnn_attention_mass_workspace_bytes(bytes(wide))
    assert need > 0 and need % 256 == 0
    assert call_mass(wide, ws=None) == E_WORKSPACE and call_mass(wide, ws=C.c_void_p((1 << 20) + 16)) == E_WORKSPACE


def test_attention_mass_workspace_stays_small():
    L = _lib.load()
    assert L.ftcnn_attention_mass_workspace_bytes(bytes(mass())) == 0 and L.ftcnn_attention_mass_workspace_bytes(None) == 0
    for kw in (dict(list_len=2**26, max_kv=0), dict(batch=4096, tokens=4096 * 40, list_len=8192, max_q=40, max_kv=0),
               dict(batch=1, tokens=1 << 20, max_q=0, list_len=2**26, max_kv=0), dict(batch=1 << 20, tokens=1 << 22, max_q=40)):
        assert L.ftcnn_attention_mass_workspace_bytes(bytes(mass(kw))) <= 1 << 28


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), E_DTYPE), (dict(batch=-1), E_SHAPE), (dict(kv_heads=0), E_SHAPE), (dict(pages=0), E_SHAPE),
    (dict(page=0), E_SHAPE), (dict(list_len=-1), E_SHAPE), (dict(max_kv=-1), E_SHAPE), (dict(first=-1), E_ARG),
    (dict(dim=4), E_UNSUPPORTED), (dict(dim=20), E_UNSUPPORTED), (dict(dim=512), E_UNSUPPORTED), (dict(list_len=2**30, page=2), E_SHAPE),
    (dict(batch=1 << 29, kv_heads=4), E_SHAPE), (dict(batch=1 << 23), E_SHAPE)])
def test_evict_refuses(kw, code):
    d = evict(kw)
    assert call_evict(d) == code
    assert "evict" in ft.last_error()
    assert _lib.load().ftcnn_evict_workspace_bytes(bytes(d)) == 0


@pytest.mark.parametrize("kw", [{("k_cache_stride", 1): 68}, {("v_cache_stride", 0): -2048}, {("v_cache_stride", 2): (1 << 29) + 8},
                                dict(mass_out_stride=79), dict(position_out_stride=0)])
def test_evict_refuses_strides(kw):
    assert call_evict(evict(kw)) == E_UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(lists=None), dict(lens=None), dict(keep=None), dict(m=None),
                                dict(lo=None), dict(mo=None), dict(po=None)])
def test_evict_refuses_missing_pointers(kw):
    assert call_evict(evict(), **kw) == E_ARG


def test_evict_refuses_what_does_not_fit():
    assert call_evict(evict(), k=ODD) == E_UNSUPPORTED and call_evict(evict(), v=ODD) == E_UNSUPPORTED
    assert call_evict(evict(dict(mass_stride=96))) == E_ARG          # in place, other strides
    assert call_evict(evict(dict(position_stride=96))) == E_ARG
    assert call_evict(evict(), ws=None) == E_WORKSPACE and call_evict(evict(), ws=C.c_void_p((1 << 20) + 16)) == E_WORKSPACE
    need = _lib.load().ftcnn_evict_workspace_bytes(bytes(evict()))
    assert need % 256 == 0 and need >= 2 * 80 * 4 and _lib.load().ftcnn_evict_workspace_bytes(None) == 0


def test_nothing_to_do_is_no_launch():
    assert call_low_rank(low_rank(dict(tokens=0)), y=None, x=None, out=None) == 0
    assert call_mass(mass(dict(tokens=0, batch=0)), q=None, m=None) == 0
    assert call_mass(mass(dict(list_len=0)), lists=None, m=None) == 0
    assert call_evict(evict(dict(batch=0)), k=None, lo=None) == 0


def test_null_descriptors():
    L = _lib.load()
    assert L.ftcnn_low_rank_add(None, *[P] * 9, None) == E_ARG
    assert L.ftcnn_attention_mass(None, *[P] * 8, None) == E_ARG
    assert L.ftcnn_evict(None, *[P] * 12, None) == E_ARG


def test_binding_refuses_host_tensors():
    y, c, i32 = torch.zeros(2, 64), torch.zeros(3, 16, 2, 64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ft.FtcnnError, match="on a device"):
        adapters.low_rank_add(y, y, y.view(1, 2, 64), y.view(1, 64, 2), i32)
    with pytest.raises(ft.FtcnnError, match="on a device"):
        paged.attention_mass(y, c[0, :2], c, i32.view(2, 1), i32, y)
    with pytest.raises(ft.FtcnnError, match="on a device"):
        paged.evict(c, c, i32.view(2, 1), i32, i32, y)


def test_low_rank_add_takes_as_many_grouped_tokens_as_are_launched():
    """A tile of the grouped launches is a workgroup of 256 threads in the first and a quarter of one in the second: 4096 parts of
    2112 tiles are within 2^32 threads of each, 8192 of them are not."""
    sizes = dict(ch=8, m=8, adapters=7000, rank=8, x_stride=8, y_stride=8, out_stride=8)
    assert _lib.load().ftcnn_low_rank_workspace_bytes(bytes(low_rank(dict(sizes, tokens=1 << 23)))) > (1 << 23) * 8 * 4
    assert call_low_rank(low_rank(dict(sizes, tokens=1 << 23)), ws=None) == E_WORKSPACE
    assert call_low_rank(low_rank(dict(sizes, tokens=1 << 24))) == E_SHAPE


@pytest.mark.parametrize("kw", [dict(kv_heads=(1 << 29) + 1, dim=8), dict(kv_heads=1 << 30, dim=8), dict(kv_heads=1 << 24, dim=256, dtype=0)])
def test_evict_refuses_rows_of_more_units_than_it_counts(kw):
    """A row of all key heads, keys and values, is counted in 16-byte units in 31 bits."""
    assert call_evict(evict(dict(kw, batch=1))) == E_SHAPE
    assert "evict" in ft.last_error()
