"""The serving operators' C entry points and binding at the ends of their arguments' ranges, on the host (no GPU
needed)."""
import pytest

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import _lib
from test_paged_abi import E_SHAPE, attention, call_attention


@pytest.mark.parametrize("kw", [dict(batch=0, tokens=4), dict(batch=0, tokens=4, max_q=0, max_kv=0),
                                dict(batch=0, tokens=4, window=7), dict(batch=4, tokens=0), dict(batch=0, tokens=0)])
def test_no_sequences_or_no_queries_take_no_room(kw):
    assert _lib.load().ftcnn_paged_attention_workspace_bytes(bytes(attention(**kw))) == 0


def test_more_key_heads_than_the_plan_counts_are_refused():
    """2^31 units of 2^30 keys and their like: their product passes 64 bits."""
    big = attention(batch=2 ** 31 - 1, tokens=1, heads=2 ** 30, kv_heads=2 ** 30, list_len=2 ** 26, max_q=0, max_kv=0)
    assert _lib.load().ftcnn_paged_attention_workspace_bytes(bytes(big)) == 0
    assert call_attention(big) == E_SHAPE
    assert "sequences" in ft.last_error()


@pytest.mark.parametrize("kw", [
    dict(batch=2 ** 30, tokens=1, heads=1, kv_heads=1), dict(batch=1, tokens=1, heads=2 ** 30, kv_heads=2 ** 30),
    dict(batch=2 ** 15, tokens=2 ** 15, heads=2 ** 15, kv_heads=2 ** 15), dict(batch=1, tokens=2 ** 30, heads=1, kv_heads=1),
    dict(batch=2 ** 30, tokens=2 ** 30, heads=1, kv_heads=1)])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("hints", [(0, 0), (1, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_the_largest_sizes_have_a_plan(kw, dtype, hints):
    d = attention(dtype=dtype, list_len=2 ** 26, max_q=hints[0], max_kv=hints[1], **kw)
    assert _lib.load().ftcnn_paged_attention_workspace_bytes(bytes(d)) < 1 << 32
