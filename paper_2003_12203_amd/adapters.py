"""Low-rank adapters of many requests beside a projection that they share.

A projection is a layer of 1x1 maps with the tokens as the batch (``Layer(tokens, ch, 1, 1, m, 1, 1)``); its
output [tokens][m] comes first, and every token's own adapter is added to it:

    y = layer.empty_output()
    layer.protected_fused(x, w, y)
    out = adapters.low_rank_add(y.view(tokens, m), x.view(tokens, ch), a, b, ids, scales)

The function has the name of the C entry point of ``include/ftcnn.h``, which gives its formula, limits and
treatment of indices, and only checks and marshals arguments, like those of ``paged``.  It is not
checksum-protected and has no backward pass.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from . import _lib
from .paged import (_CONTIGUOUS, _DTYPE, _F32, _I32, _On, _bad, _current_device, _fail, _is, _no_backward, _raw_stream,
                    _recording, _room)

_LOW_RANK = struct.Struct("=6i7q")   # the layout of _lib.LowRankDesc


def low_rank_add(y: torch.Tensor, x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor,
                 scales: Optional[torch.Tensor] = None, ranks: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """ftcnn_low_rank_add: y[t] + scales[i] * b[i] @ (a[i] @ x[t]) with i = ids[t] (int32 [tokens]; -1: no adapter).
    y [tokens][m], x [tokens][ch], a [adapters][rank][ch] and b [adapters][m][rank] are all float32 or bfloat16, strided as
    they come with the last dimension contiguous; scales float32 [adapters]; ranks int32 [adapters], where adapters use
    fewer than rank, which is a multiple of 4 (float32) or 8 (bfloat16), at most 128.  The output is allocated, contiguous,
    unless given (in place: out=y).  workspace: uint8, 256-byte aligned; allocated when not given."""
    what = "low_rank_add"
    dtype, shape, dev = y.dtype, y.shape, y.get_device()
    if dtype not in _DTYPE or len(shape) != 2 or dev < 0:
        _bad(what, f"y is float32 or bfloat16 [tokens][m] on a device, not {_is(y)}")
    if stream is not None or dev != _current_device():
        with _On(y.device, stream):
            return low_rank_add(y, x, a, b, ids, scales, ranks, out, workspace)
    if _recording() and (y.requires_grad or x.requires_grad or a.requires_grad or b.requires_grad or
                         (scales is not None and scales.requires_grad)):
        _no_backward(what)
    tokens, m = shape
    xshape, low = x.shape, a.shape
    if not (x.dtype is dtype and len(xshape) == 2 and xshape[0] == tokens and x.get_device() == dev):
        _bad(what, f"x must be {dtype} [{tokens}][ch] on device {dev}, not {_is(x)}")
    ch = xshape[1]
    if not (a.dtype is dtype and len(low) == 3 and low[2] == ch and a.get_device() == dev):
        _bad(what, f"a must be {dtype} [adapters][rank][{ch}] on device {dev}, not {_is(a)}")
    count, rank = low[0], low[1]
    if not (b.dtype is dtype and b.shape == (count, m, rank) and b.get_device() == dev):
        _bad(what, f"b must be {dtype} [{count}][{m}][{rank}] on device {dev}, not {_is(b)}")
    if not (ids.dtype is _I32 and ids.shape == (tokens,) and ids.is_contiguous() and ids.get_device() == dev):
        _bad(what, f"ids must be a contiguous int32 [{tokens}] on device {dev}, not {_is(ids)}")
    if scales is not None and not (scales.dtype is _F32 and scales.shape == (count,) and scales.is_contiguous() and
                                   scales.get_device() == dev):
        _bad(what, f"scales must be a contiguous float32 [{count}] on device {dev}, not {_is(scales)}")
    if ranks is not None and not (ranks.dtype is _I32 and ranks.shape == (count,) and ranks.is_contiguous() and
                                  ranks.get_device() == dev):
        _bad(what, f"ranks must be a contiguous int32 [{count}] on device {dev}, not {_is(ranks)}")
    if out is None:
        out = torch.empty_like(y, memory_format=_CONTIGUOUS)
    elif not (out.dtype is dtype and out.shape == shape and out.get_device() == dev):
        _bad(what, f"out must be like y, {dtype} {tuple(shape)} on device {dev}, not {_is(out)}")
    ys, xs, os, as_, bs = y.stride(), x.stride(), out.stride(), a.stride(), b.stride()
    if not ys[1] == xs[1] == os[1] == as_[2] == bs[2] == 1:
        _bad(what, "the last dimension of x, y, a, b and the output must be contiguous")
    try:
        desc = _LOW_RANK.pack(_DTYPE[dtype], tokens, ch, m, count, rank, xs[0], ys[0], os[0], as_[0], as_[1], bs[0], bs[1])
    except (struct.error, OverflowError) as e:
        _bad(what, f"a number that its field does not hold: {e}")
    L = _lib.load()
    room = _room(what, L.ftcnn_low_rank_workspace_bytes(desc), workspace, dev)
    rc = L.ftcnn_low_rank_add(desc, y.data_ptr(), x.data_ptr(), a.data_ptr(), b.data_ptr(), ids.data_ptr(),
                              None if scales is None else scales.data_ptr(), None if ranks is None else ranks.data_ptr(),
                              out.data_ptr(), None if room is None else room.data_ptr(), _raw_stream(dev))
    if rc:
        _fail(what, rc)
    return out
