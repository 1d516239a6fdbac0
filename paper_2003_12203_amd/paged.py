"""The operators of a serving attention layer: norms and rotation of queries and keys, a paged cache of
keys and values, and the attention of new tokens over it.

They stand between the projections of a transformer layer, which are layers of 1x1 maps with the
tokens as the batch (``Layer(tokens, ch, 1, 1, m, 1, 1)``: checksum-protected matrix products).  The
functions have the names of the C entry points of ``include/ftcnn.h``, which gives each one's formula,
limits and treatment of indices, and only check and marshal arguments; every step runs in the
library's HIP kernels, on the current torch stream or the one given.  Outputs and workspaces that a
call allocates belong to that stream.

Shapes: queries [tokens][heads][dim], keys and values [tokens][kv_heads][dim], caches
[pages][page][kv_heads][dim], of float32 or bfloat16, strided as they come with ``dim`` contiguous (a
slice of a packed projection, a cache that holds a page's heads one after the other).  There are no
backward passes: where gradients are recorded (not under ``torch.no_grad()``), a tensor that requires them is refused.

    table = paged.rope_table(max_pos, dim)
    cache = paged.PagedCache(pages, page, kv_heads, dim, "bf16")
    q, _ = paged.qk_norm_rope(q, None, positions, table, q_weight)
    paged.kv_append(k, v, cache.k, cache.v, slots, positions, table, k_weight)
    out = paged.paged_attention(q, cache.k, cache.v, page_list, kv_lens, q_starts, max_q, max_kv)
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Tuple

import torch

from . import BF16, DTYPES, F32, FtcnnError, _check, _lib

LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}
_F32, _BF16, _I32, _I64, _U8 = torch.float32, torch.bfloat16, torch.int32, torch.int64, torch.uint8
_DTYPE = {_F32: F32, _BF16: BF16}
_CONTIGUOUS = torch.contiguous_format

# the descriptors in the layout of _lib.RopeDesc, AppendDesc and AttentionDesc
_ROPE = struct.Struct("=9if8q")
_APPEND = struct.Struct("=10ifi10q")
_ATTENTION = struct.Struct("=13if11q")

# A decode step makes these calls for every layer and token, so what they cost on the host counts: a
# tensor's checks are one expression each, and the stream is asked for without a Stream object
# (0.1 us; torch.cuda.current_stream() 2.7) where torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_recording = torch.is_grad_enabled


def _bad(what: str, why: str):
    raise FtcnnError(f"{what}: {why}")


def _is(t) -> str:
    return (f"{t.dtype} {tuple(t.shape)} of strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor)
            else repr(t))


class _On:
    """The device of a call's tensors and the stream it was given made current: allocations and the launch
    go there."""

    def __init__(self, device: torch.device, stream):
        self.contexts = [torch.cuda.device(device)] + ([torch.cuda.stream(stream)] if stream is not None else [])

    def __enter__(self):
        for c in self.contexts:
            c.__enter__()

    def __exit__(self, *exc):
        for c in reversed(self.contexts):
            c.__exit__(*exc)


def _no_backward(what: str):
    _bad(what, "no backward pass: call it under torch.no_grad(), or detach the tensors that require gradients")


def _fail(what: str, rc: int):
    _check(rc, "ftcnn_" + what)


def rope_table(max_pos: int, rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
               original: int = 0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0, device="cuda",
               stream=None) -> torch.Tensor:
    """ftcnn_rope_table: (cos, sin) of every position and pair, float32 [max_pos][rot / 2][2].  scaling
    "linear", "base" or "parts" with a factor stretches the angles for longer contexts ("parts" also takes
    original, low and high)."""
    if scaling not in SCALINGS:
        _bad("rope_table", f"scaling {scaling!r}: one of {sorted(SCALINGS)}")
    if not (0 < max_pos < 1 << 31 and 2 <= rot <= 256 and rot % 2 == 0):
        _bad("rope_table", f"max_pos {max_pos}, rot {rot} (even, at most 256)")
    sc = _lib.RopeScaling(max_pos, rot, SCALINGS[scaling], original, base, factor, low, high, amplitude)
    with _On(torch.device(device), stream):
        table = torch.empty(max_pos, rot // 2, 2, dtype=_F32, device=device)
        _fail("rope_table", _lib.load().ftcnn_rope_table(C.byref(sc), table.data_ptr(),
                                                         torch.cuda.current_stream().cuda_stream))
    return table


def _rotation(what, dtype, tokens, dim, dev, positions, table, w0, w1, layout):
    """(rot, layout, max_pos, weight dtype) of a call on [tokens][heads][dim] of a dtype on device dev."""
    rot = max_pos = 0
    if table is not None:
        shape = table.shape
        if not (len(shape) == 3 and shape[2] == 2 and table.dtype is _F32 and table.is_contiguous() and
                table.get_device() == dev):
            _bad(what, f"the table must be a contiguous float32 [max_pos][rot / 2][2] on device {dev}, not {_is(table)}")
        if positions is None or not (positions.dtype is _I32 and positions.shape == (tokens,) and
                                     positions.is_contiguous() and positions.get_device() == dev):
            _bad(what, f"positions must be a contiguous int32 [{tokens}] on device {dev}, not {_is(positions)}")
        max_pos, rot = shape[0], 2 * shape[1]
    elif positions is not None:
        _bad(what, "positions need a table")
    if layout not in LAYOUTS:
        _bad(what, f"layout {layout!r}: one of {sorted(LAYOUTS)}")
    wd = None
    for w in (w0, w1):
        if w is not None:
            if not (w.shape == (dim,) and w.is_contiguous() and w.get_device() == dev and
                    (w.dtype is dtype or w.dtype is _F32) and (wd is None or wd is w.dtype)):
                _bad(what, f"weights must be contiguous [{dim}] of float32 or {dtype}, both alike, on device {dev}, "
                           f"not {_is(w)}")
            wd = w.dtype
    return rot, LAYOUTS[layout], max_pos, F32 if wd is None else _DTYPE[wd]


def qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                 table: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, layout: str = "half",
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                 stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """ftcnn_qk_norm_rope: queries and keys normed for each head (with a weight [dim]) and rotated by position
    (positions int32 [tokens], table of rope_table).  Either may be None.  Outputs are allocated, contiguous,
    unless given (in place: q_out=q)."""
    what = "qk_norm_rope"
    x = q if q is not None else k
    if x is None:
        _bad(what, "neither queries nor keys")
    dtype, shape, dev = x.dtype, x.shape, x.get_device()
    if dtype not in _DTYPE or len(shape) != 3 or dev < 0:
        _bad(what, f"queries and keys are float32 or bfloat16 [tokens][heads][dim] on a device, not {_is(x)}")
    if stream is not None or dev != _current_device():
        with _On(x.device, stream):
            return qk_norm_rope(q, k, positions, table, q_weight, k_weight, eps, layout, q_out, k_out)
    if _recording() and (x.requires_grad or (k is not None and k.requires_grad) or
                         (q_weight is not None and q_weight.requires_grad) or
                         (k_weight is not None and k_weight.requires_grad)):
        _no_backward(what)
    tokens, heads, dim = shape
    kv_heads = 0
    rot, lay, max_pos, wd = _rotation(what, dtype, tokens, dim, dev, positions, table, q_weight, k_weight, layout)
    qi = qo = ki = ko = (0, 0, 1)
    if q is None:
        heads, q_out = 0, None
    else:
        qi = q.stride()
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=_CONTIGUOUS)
        elif not (q_out.dtype is dtype and q_out.shape == shape and q_out.get_device() == dev):
            _bad(what, f"q_out must be like q, not {_is(q_out)}")
        qo = q_out.stride()
    if k is None:
        k_out = None
    else:
        ki, kshape = k.stride(), k.shape
        if not (k.dtype is dtype and len(kshape) == 3 and kshape[0] == tokens and kshape[2] == dim and
                k.get_device() == dev):
            _bad(what, f"k must be {dtype} [{tokens}][kv_heads][{dim}] on device {dev}, not {_is(k)}")
        kv_heads = kshape[1]
        if k_out is None:
            k_out = torch.empty_like(k, memory_format=_CONTIGUOUS)
        elif not (k_out.dtype is dtype and k_out.shape == kshape and k_out.get_device() == dev):
            _bad(what, f"k_out must be like k, not {_is(k_out)}")
        ko = k_out.stride()
    if not qi[2] == qo[2] == ki[2] == ko[2] == 1:
        _bad(what, "the last dimension of queries, keys and outputs must be contiguous")
    try:
        desc = _ROPE.pack(_DTYPE[dtype], tokens, heads, kv_heads, dim, rot, lay, max_pos, wd, eps, qi[0], qi[1], ki[0],
                          ki[1], qo[0], qo[1], ko[0], ko[1])
    except (struct.error, OverflowError) as e:
        _bad(what, f"a number that its field does not hold: {e}")
    rc = _lib.load().ftcnn_qk_norm_rope(
        desc, None if q is None else q.data_ptr(), None if k is None else k.data_ptr(),
        None if positions is None else positions.data_ptr(), None if table is None else table.data_ptr(),
        None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
        None if q is None else q_out.data_ptr(), None if k is None else k_out.data_ptr(), _raw_stream(dev))
    if rc:
        _fail(what, rc)
    return q_out, k_out


def kv_append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, slots: torch.Tensor,
              positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, layout: str = "half",
              stream=None) -> None:
    """ftcnn_kv_append: the new tokens' keys (normed with a weight, rotated with positions and a table) and
    values into the cache rows slots (int64 [tokens], page * rows of a page + row; -1: nowhere)."""
    what = "kv_append"
    dtype, shape, dev = k.dtype, k.shape, k.get_device()
    if dtype not in _DTYPE or len(shape) != 3 or dev < 0:
        _bad(what, f"keys are float32 or bfloat16 [tokens][kv_heads][dim] on a device, not {_is(k)}")
    if stream is not None or dev != _current_device():
        with _On(k.device, stream):
            return kv_append(k, v, k_cache, v_cache, slots, positions, table, k_weight, eps, layout)
    if _recording() and (k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad or
                         (k_weight is not None and k_weight.requires_grad)):
        _no_backward(what)
    tokens, kv_heads, dim = shape
    if not (v.dtype is dtype and v.shape == shape and v.get_device() == dev):
        _bad(what, f"v must be like k, {dtype} {tuple(shape)} on device {dev}, not {_is(v)}")
    cache = k_cache.shape
    if not (k_cache.dtype is dtype and len(cache) == 4 and cache[2] == kv_heads and cache[3] == dim and
            k_cache.get_device() == dev):
        _bad(what, f"k_cache must be {dtype} [pages][page][{kv_heads}][{dim}] on device {dev}, not {_is(k_cache)}")
    if not (v_cache.dtype is dtype and v_cache.shape == cache and v_cache.get_device() == dev):
        _bad(what, f"v_cache must be like k_cache, {dtype} {tuple(cache)} on device {dev}, not {_is(v_cache)}")
    if not (slots.dtype is _I64 and slots.shape == (tokens,) and slots.is_contiguous() and slots.get_device() == dev):
        _bad(what, f"slots must be a contiguous int64 [{tokens}] on device {dev}, not {_is(slots)}")
    rot, lay, max_pos, wd = _rotation(what, dtype, tokens, dim, dev, positions, table, k_weight, None, layout)
    ks, vs, kc, vc = k.stride(), v.stride(), k_cache.stride(), v_cache.stride()
    if not ks[2] == vs[2] == kc[3] == vc[3] == 1:
        _bad(what, "the last dimension of keys, values and caches must be contiguous")
    try:
        desc = _APPEND.pack(_DTYPE[dtype], tokens, kv_heads, dim, rot, lay, max_pos, wd, cache[0], cache[1], eps, 0,
                            ks[0], ks[1], vs[0], vs[1], kc[0], kc[1], kc[2], vc[0], vc[1], vc[2])
    except (struct.error, OverflowError) as e:
        _bad(what, f"a number that its field does not hold: {e}")
    rc = _lib.load().ftcnn_kv_append(
        desc, k.data_ptr(), v.data_ptr(), None if positions is None else positions.data_ptr(),
        None if table is None else table.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
        slots.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _raw_stream(dev))
    if rc:
        _fail(what, rc)


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_list: torch.Tensor,
                    kv_lens: torch.Tensor, q_starts: Optional[torch.Tensor] = None, max_q: int = 0, max_kv: int = 0,
                    scale: Optional[float] = None, causal: bool = True, window: int = 0,
                    out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ftcnn_paged_attention: the new tokens q [tokens][heads][dim] of a batch of sequences over each one's
    pages (page_list int32 [batch][entries], kv_lens int32 [batch], the new tokens' rows among them).
    q_starts int32 [batch + 1] says whose tokens are whose (None: one of each sequence; tokens of no sequence are
    0).  max_q and max_kv, the
    longest sequence's new and cached tokens where the caller knows them, size the launch (and, in bf16, max_q decides
    which calls round their softmax weights).  scale defaults to
    1 / sqrt(dim).  lse (float32 [tokens][heads]) is filled when given.  workspace: uint8, 256-byte aligned;
    allocated when needed and not given."""
    what = "paged_attention"
    dtype, shape, dev = q.dtype, q.shape, q.get_device()
    if dtype not in _DTYPE or len(shape) != 3 or dev < 0:
        _bad(what, f"queries are float32 or bfloat16 [tokens][heads][dim] on a device, not {_is(q)}")
    if stream is not None or dev != _current_device():
        with _On(q.device, stream):
            return paged_attention(q, k_cache, v_cache, page_list, kv_lens, q_starts, max_q, max_kv, scale, causal,
                                   window, out, lse, workspace)
    if _recording() and (q.requires_grad or k_cache.requires_grad or v_cache.requires_grad):
        _no_backward(what)
    tokens, heads, dim = shape
    cache = k_cache.shape
    if not (k_cache.dtype is dtype and len(cache) == 4 and cache[3] == dim and k_cache.get_device() == dev):
        _bad(what, f"k_cache must be {dtype} [pages][page][kv_heads][{dim}] on device {dev}, not {_is(k_cache)}")
    if not (v_cache.dtype is dtype and v_cache.shape == cache and v_cache.get_device() == dev):
        _bad(what, f"v_cache must be like k_cache, {dtype} {tuple(cache)} on device {dev}, not {_is(v_cache)}")
    lists = page_list.shape
    if not (page_list.dtype is _I32 and len(lists) == 2 and (page_list.stride(1) == 1 or lists[1] < 2) and
            page_list.get_device() == dev):
        _bad(what, f"page_list must be int32 [batch][entries], entries contiguous, on device {dev}, not "
                   f"{_is(page_list)}")
    batch, entries = lists
    if not (kv_lens.dtype is _I32 and kv_lens.shape == (batch,) and kv_lens.is_contiguous() and
            kv_lens.get_device() == dev):
        _bad(what, f"kv_lens must be a contiguous int32 [{batch}] on device {dev}, not {_is(kv_lens)}")
    if q_starts is not None and not (q_starts.dtype is _I32 and q_starts.shape == (batch + 1,) and
                                     q_starts.is_contiguous() and q_starts.get_device() == dev):
        _bad(what, f"q_starts must be a contiguous int32 [{batch + 1}] on device {dev}, not {_is(q_starts)}")
    if q_starts is None:
        max_q = 1
    if lse is not None and not (lse.dtype is _F32 and lse.shape == (tokens, heads) and lse.is_contiguous() and
                                lse.get_device() == dev):
        _bad(what, f"lse must be a contiguous float32 [{tokens}][{heads}] on device {dev}, not {_is(lse)}")
    if out is None:
        out = torch.empty_like(q, memory_format=_CONTIGUOUS)
    elif not (out.dtype is dtype and out.shape == shape and out.get_device() == dev):
        _bad(what, f"out must be like q, {dtype} {tuple(shape)} on device {dev}, not {_is(out)}")
    qs, os, kc, vc = q.stride(), out.stride(), k_cache.stride(), v_cache.stride()
    if not qs[2] == os[2] == kc[3] == vc[3] == 1:
        _bad(what, "the last dimension of queries, caches and outputs must be contiguous")
    if scale is None:
        scale = dim ** -0.5 if dim else 1.0   # (no dim: refused with the other sizes)
    try:
        desc = _ATTENTION.pack(_DTYPE[dtype], batch, tokens, heads, cache[2], dim, cache[0], cache[1], entries, causal,
                               window, max_q, max_kv, scale, qs[0], qs[1], os[0], os[1],
                               kc[0], kc[1], kc[2], vc[0], vc[1], vc[2], page_list.stride(0))
    except (struct.error, OverflowError) as e:
        _bad(what, f"a number that its field does not hold: {e}")
    L = _lib.load()
    need = L.ftcnn_paged_attention_workspace_bytes(desc)
    room = None
    if need:
        if workspace is None:
            workspace = torch.empty(need, dtype=_U8, device=q.device)
        elif not (workspace.dtype is _U8 and workspace.numel() >= need and workspace.is_contiguous() and
                  workspace.get_device() == dev):
            _bad(what, f"the workspace must be {need} contiguous bytes on device {dev}, not {_is(workspace)}")
        room = workspace.data_ptr()
    rc = L.ftcnn_paged_attention(desc, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), page_list.data_ptr(),
                                 kv_lens.data_ptr(), None if q_starts is None else q_starts.data_ptr(),
                                 out.data_ptr(), None if lse is None else lse.data_ptr(), room, _raw_stream(dev))
    if rc:
        _fail(what, rc)
    return out


class PagedCache:
    """The keys and values of one layer in pages: k and v [pages][page][kv_heads][dim], each page's heads one
    after the other in memory (a head's rows of a page are one run)."""

    def __init__(self, pages: int, page: int, kv_heads: int, dim: int, dtype: str = "bf16", device="cuda"):
        shape = (pages, kv_heads, page, dim)
        dt = DTYPES[dtype][1]
        self.k = torch.zeros(shape, dtype=dt, device=device).transpose(1, 2)
        self.v = torch.zeros(shape, dtype=dt, device=device).transpose(1, 2)
        self.pages, self.page = pages, page

    def slots(self, page_list: torch.Tensor, seq: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """The rows (for kv_append) of tokens at the given positions of sequences seq; -1 (written nowhere) for padding:
        a sequence or position outside the list."""
        batch, entries = page_list.shape
        p, s = positions.long(), seq.long()
        if batch * entries == 0:
            return torch.full_like(p, -1)
        p_in, s_in = p.clamp(0, entries * self.page - 1), s.clamp(0, batch - 1)
        rows = page_list[s_in, p_in // self.page].long() * self.page + p_in % self.page
        return torch.where((p == p_in) & (s == s_in), rows, -1)
