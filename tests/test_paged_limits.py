"""The serving operators' C entry points and binding at the ends of their arguments' ranges, on the host (no GPU
needed)."""
import pytest
import torch

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import _lib, paged
from test_paged_abi import E_ARG, E_SHAPE, attention, call_attention


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


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_rows_of_padding_are_nowhere(dtype):
    """Positions and sequences outside the list have no row: no other token's either."""
    cache = paged.PagedCache(6, 4, 2, 8, "f32", device="cpu")
    lists = torch.tensor([[5, 1, 0], [2, 3, 4]], dtype=torch.int32)
    seq = torch.tensor([0, 0, 0, 0, 1, 1, -1, 2, 1, -1], dtype=dtype)
    pos = torch.tensor([-1, 0, 11, 12, -7, 2 ** 31 - 1, 3, 3, 5, -1], dtype=dtype)
    got = cache.slots(lists, seq, pos)
    assert got.dtype == torch.int64
    assert got.tolist() == [-1, 20, 3, -1, -1, -1, -1, -1, 13, -1]
    assert cache.slots(lists[:, :0], seq, pos).tolist() == [-1] * 10
    assert cache.slots(lists[:0], seq, pos).tolist() == [-1] * 10
    # entries of a list that name no page
    gone = torch.tensor([[-1, 6]], dtype=torch.int32)
    at = cache.slots(gone, torch.zeros(8, dtype=dtype), torch.arange(8, dtype=dtype))
    assert ((at < 0) | (at >= 24)).all()


def test_a_scale_that_overflows_in_powers_of_two_is_refused():
    assert call_attention(attention(scale=3e38)) == E_ARG
    assert "scale" in ft.last_error()
