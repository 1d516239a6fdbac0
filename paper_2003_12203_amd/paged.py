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
slice of a packed projection, a cache that holds a page's heads one after the other).

    table = paged.rope_table(max_pos, dim)
    cache = paged.PagedCache(pages, page, kv_heads, dim, "bf16")
    q, _ = paged.qk_norm_rope(q, None, positions, table, q_weight)
    paged.kv_append(k, v, cache.k, cache.v, slots, positions, table, k_weight)
    out = paged.paged_attention(q, cache.k, cache.v, page_list, kv_lens, q_starts, max_q, max_kv)
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional, Tuple

import torch

from . import BF16, DTYPES, F32, FtcnnError, _check, _lib

LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}
_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}

# the descriptors in the layout of _lib.RopeDesc, AppendDesc and AttentionDesc
_ROPE = struct.Struct("=9if8q")
_APPEND = struct.Struct("=10ifi10q")
_ATTENTION = struct.Struct("=13if11q")


def _bad(what: str, why: str):
    raise FtcnnError(f"{what}: {why}")


def _tensor(what: str, name: str, t: torch.Tensor, dims: int, dtype=None, like: Optional[torch.Tensor] = None):
    if t.dim() != dims:
        _bad(what, f"{name} must have {dims} dimensions, not {t.dim()}")
    if dtype is not None and t.dtype != dtype:
        _bad(what, f"{name} must be {dtype}, not {t.dtype}")
    if like is None:
        if not t.is_cuda:
            _bad(what, f"{name} must be a device tensor")
    elif t.device != like.device:
        _bad(what, f"{name} is on {t.device}, not on {like.device}")


def _heads(what: str, name: str, t: torch.Tensor, dims: int, dtype, like):
    """A tensor of heads: its last dimension contiguous."""
    _tensor(what, name, t, dims, dtype, like)
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        _bad(what, f"the last dimension of {name} must be contiguous")


def _vector(what: str, name: str, t: torch.Tensor, n: int, dtype, like):
    _tensor(what, name, t, 1, dtype, like)
    if t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        _bad(what, f"{name} must be a contiguous vector of {n}, not {tuple(t.shape)}")


class _On:
    """The device and stream of a call: allocations and the launch go there."""

    def __init__(self, device: torch.device, stream):
        self.given = torch.cuda.stream(stream) if stream is not None else None
        self.device = torch.cuda.device(device) if device.index not in (None, torch.cuda.current_device()) else None

    def __enter__(self):
        if self.device is not None:
            self.device.__enter__()
        if self.given is not None:
            self.given.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        if self.given is not None:
            self.given.__exit__(*exc)
        if self.device is not None:
            self.device.__exit__(*exc)


def rope_table(max_pos: int, rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
               original: int = 0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0, device="cuda",
               stream=None) -> torch.Tensor:
    """ftcnn_rope_table: (cos, sin) of every position and pair, float32 [max_pos][rot / 2][2].  scaling
    "linear", "base" or "parts" with a factor stretches the angles for longer contexts ("parts" also takes
    original, low and high)."""
    if scaling not in SCALINGS:
        _bad("rope_table", f"scaling {scaling!r}: one of {sorted(SCALINGS)}")
    sc = _lib.RopeScaling(max_pos, rot, SCALINGS[scaling], original, base, factor, low, high, amplitude)
    if not (0 < max_pos < 1 << 31 and 2 <= rot <= 256 and rot % 2 == 0):
        _bad("rope_table", f"max_pos {max_pos}, rot {rot} (even, at most 256)")
    with _On(torch.device(device), stream) as st:
        table = torch.empty(max_pos, rot // 2, 2, dtype=torch.float32, device=device)
        _check(_lib.load().ftcnn_rope_table(C.byref(sc), table.data_ptr(), st), "ftcnn_rope_table")
    return table


def _rotation(what, x, positions, table, layout, weights):
    """(rot, layout, max_pos, weight dtype) of a call on x [tokens][heads][dim]."""
    if (positions is None) != (table is None):
        _bad(what, "positions and table go together")
    rot = max_pos = 0
    if table is not None:
        _vector(what, "positions", positions, x.shape[0], torch.int32, x)
        _tensor(what, "table", table, 3, torch.float32, x)
        if table.shape[2] != 2 or not table.is_contiguous():
            _bad(what, f"the table must be a contiguous [max_pos][rot / 2][2], not {tuple(table.shape)}")
        max_pos, rot = table.shape[0], 2 * table.shape[1]
    if layout not in LAYOUTS:
        _bad(what, f"layout {layout!r}: one of {sorted(LAYOUTS)}")
    wd = None
    for w in weights:
        if w is not None:
            _vector(what, "a weight", w, x.shape[2], None, x)
            if w.dtype not in (torch.float32, x.dtype) or (wd is not None and w.dtype != wd):
                _bad(what, f"weights must be float32 or {x.dtype}, both the same")
            wd = w.dtype
    return rot, LAYOUTS[layout], max_pos, F32 if wd is None else _DTYPE[wd]


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


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
    if x.dtype not in _DTYPE:
        _bad(what, f"dtype {x.dtype}")
    for name, t in (("q", q), ("k", k)):
        if t is not None:
            _heads(what, name, t, 3, x.dtype, None if t is x else x)
            if t.shape[0] != x.shape[0] or t.shape[2] != x.shape[2]:
                _bad(what, "q and k must agree on tokens and dim")
    rot, lay, max_pos, wd = _rotation(what, x, positions, table, layout, (q_weight, k_weight))
    tokens, _, dim = x.shape
    with _On(x.device, stream) as st:
        outs, hd, si, so = [], [], [], []
        for name, t, o in (("q_out", q, q_out), ("k_out", k, k_out)):
            if t is None:
                outs.append(None)
                hd.append(0)
                si += (0, 0)
                so += (0, 0)
                continue
            if o is None:
                o = torch.empty(t.shape, dtype=t.dtype, device=t.device)
            else:
                _heads(what, name, o, 3, t.dtype, x)
                if o.shape != t.shape:
                    _bad(what, f"{name} must be {tuple(t.shape)}, not {tuple(o.shape)}")
            outs.append(o)
            hd.append(t.shape[1])
            si += t.stride()[:2]
            so += o.stride()[:2]
        desc = _ROPE.pack(_DTYPE[x.dtype], tokens, hd[0], hd[1], dim, rot, lay, max_pos, wd, eps, *si, *so)
        _check(_lib.load().ftcnn_qk_norm_rope(desc, _at(q), _at(k), _at(positions), _at(table), _at(q_weight),
                                              _at(k_weight), _at(outs[0]), _at(outs[1]), st), "ftcnn_qk_norm_rope")
    return outs[0], outs[1]


def _caches(what, k_cache, v_cache, like, kv_heads, dim):
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _heads(what, name, t, 4, like.dtype, like)
    shape = k_cache.shape
    if v_cache.shape != shape or shape[3] != dim or (kv_heads is not None and shape[2] != kv_heads):
        _bad(what, f"caches of {tuple(shape)} and {tuple(v_cache.shape)} for heads of {dim}")
    return shape


def kv_append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, slots: torch.Tensor,
              positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, layout: str = "half",
              stream=None) -> None:
    """ftcnn_kv_append: the new tokens' keys (normed with a weight, rotated with positions and a table) and
    values into the cache rows slots (int64 [tokens], page * rows of a page + row; -1: nowhere)."""
    what = "kv_append"
    if k.dtype not in _DTYPE:
        _bad(what, f"dtype {k.dtype}")
    _heads(what, "k", k, 3, None, None)
    _heads(what, "v", v, 3, k.dtype, k)
    if v.shape != k.shape:
        _bad(what, f"k {tuple(k.shape)} and v {tuple(v.shape)} must agree")
    tokens, kv_heads, dim = k.shape
    pages, page = _caches(what, k_cache, v_cache, k, kv_heads, dim)[:2]
    _vector(what, "slots", slots, tokens, torch.int64, k)
    rot, lay, max_pos, wd = _rotation(what, k, positions, table, layout, (k_weight,))
    with _On(k.device, stream) as st:
        desc = _APPEND.pack(_DTYPE[k.dtype], tokens, kv_heads, dim, rot, lay, max_pos, wd, pages, page, eps, 0,
                            *k.stride()[:2], *v.stride()[:2], *k_cache.stride()[:3], *v_cache.stride()[:3])
        _check(_lib.load().ftcnn_kv_append(desc, _at(k), _at(v), _at(positions), _at(table), _at(k_weight),
                                           _at(slots), _at(k_cache), _at(v_cache), st), "ftcnn_kv_append")


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_list: torch.Tensor,
                    kv_lens: torch.Tensor, q_starts: Optional[torch.Tensor] = None, max_q: int = 0, max_kv: int = 0,
                    scale: Optional[float] = None, causal: bool = True, window: int = 0,
                    out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ftcnn_paged_attention: the new tokens q [tokens][heads][dim] of a batch of sequences over each one's
    pages (page_list int32 [batch][entries], kv_lens int32 [batch], the new tokens' rows among them).
    q_starts int32 [batch + 1] says whose tokens are whose (None: one of each sequence).  max_q and max_kv, the
    longest sequence's new and cached tokens where the caller knows them, size the launch.  scale defaults to
    1 / sqrt(dim).  lse (float32 [tokens][heads]) is filled when given.  workspace: uint8, 256-byte aligned,
    of attention_workspace_bytes; allocated when needed and not given."""
    what = "paged_attention"
    if q.dtype not in _DTYPE:
        _bad(what, f"dtype {q.dtype}")
    _heads(what, "q", q, 3, None, None)
    tokens, heads, dim = q.shape
    pages, page, kv_heads, _ = _caches(what, k_cache, v_cache, q, None, dim)
    _tensor(what, "page_list", page_list, 2, torch.int32, q)
    batch, entries = page_list.shape
    if entries > 1 and page_list.stride(1) != 1:
        _bad(what, "the last dimension of page_list must be contiguous")
    _vector(what, "kv_lens", kv_lens, batch, torch.int32, q)
    if q_starts is not None:
        _vector(what, "q_starts", q_starts, batch + 1, torch.int32, q)
    if lse is not None:
        _tensor(what, "lse", lse, 2, torch.float32, q)
        if lse.shape != q.shape[:2] or not lse.is_contiguous():
            _bad(what, f"lse must be a contiguous {tuple(q.shape[:2])}")
    if out is not None:
        _heads(what, "out", out, 3, q.dtype, q)
        if out.shape != q.shape:
            _bad(what, f"out must be {tuple(q.shape)}, not {tuple(out.shape)}")
    with _On(q.device, stream) as st:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        desc = _ATTENTION.pack(_DTYPE[q.dtype], batch, tokens, heads, kv_heads, dim, pages, page, entries,
                               int(causal), window, max_q, max_kv, 1.0 / math.sqrt(dim) if scale is None else scale,
                               *q.stride()[:2], *out.stride()[:2], *k_cache.stride()[:3], *v_cache.stride()[:3],
                               page_list.stride(0))
        L = _lib.load()
        need = L.ftcnn_paged_attention_workspace_bytes(desc)
        if need:
            if workspace is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            else:
                _tensor(what, "workspace", workspace, 1, torch.uint8, q)
                if workspace.numel() < need or not workspace.is_contiguous():
                    _bad(what, f"the workspace must be {need} contiguous bytes, not {workspace.numel()}")
        _check(L.ftcnn_paged_attention(desc, _at(q), _at(k_cache), _at(v_cache), _at(page_list), _at(kv_lens),
                                       _at(q_starts), _at(out), _at(lse), _at(workspace) if need else None, st),
               "ftcnn_paged_attention")
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
        """The rows (for kv_append) of tokens at the given positions of sequences seq."""
        p = positions.long()
        return page_list[seq.long(), p // self.page].long() * self.page + p % self.page
