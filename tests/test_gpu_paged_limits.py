"""Attention over the paged cache at the ends of its arguments' ranges, against its definition in float64."""
import numpy as np
import pytest

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import paged
from test_gpu_paged import batch, check

pytestmark = pytest.mark.gpu


def is_split(q, kc, lists, new, length, **kw):
    """Whether the call takes even runs (and room for their parts)."""
    d = ft._lib.AttentionDesc(paged._DTYPE[q.dtype], lists.shape[0], q.shape[0], q.shape[1], kc.shape[2], q.shape[2],
                              kc.shape[0], kc.shape[1], lists.shape[1], kw.get("causal", 1), kw.get("window", 0),
                              max(new), max(length), 1.0)
    return ft._lib.load().ftcnn_paged_attention_workspace_bytes(bytes(d)) > 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 20, 2 ** 30, 6017])
@pytest.mark.parametrize("new,length,split", [
    ([200], [6000], True),                  # a chunk whose keys are split over workgroups
    ([1, 4], [6000, 2000], True),           # single tokens and a few, by single waves
    ([60, 20, 3], [60, 12, 0], False)])     # whole units; more new tokens than cached
def test_windows_wider_than_any_sequence(dtype, window, new, length, split):
    rng = np.random.default_rng(window % 1000)
    args = batch(rng, new, length, 4, 1, 64, dtype, 16, fill=float("nan"))
    assert is_split(args[0], args[1], args[3], new, length, window=window) == split
    check(*args, dtype, window=window, max_q=max(new), max_kv=max(length))
