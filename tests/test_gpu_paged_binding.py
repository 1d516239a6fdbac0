"""What the Python binding of the serving operators refuses."""
import importlib.util

import pytest
import torch

import paper_2003_12203_amd as ft
from paper_2003_12203_amd import paged

pytestmark = pytest.mark.gpu


def arguments(dtype=torch.bfloat16):
    """One sequence of five tokens, of which three are new: (queries, keys, values, caches, arrays by name)."""
    torch.manual_seed(0)
    x = torch.randn(3, 8, 64, device="cuda").to(dtype)
    cache = paged.PagedCache(2, 16, 2, 64, "bf16" if dtype is torch.bfloat16 else "f32")
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(q=x[:, :4], k=x[:, 4:6], v=x[:, 6:], k_cache=cache.k, v_cache=cache.v, table=paged.rope_table(8, 64),
                q_weight=torch.ones(64, device="cuda"), k_weight=torch.ones(64, device="cuda"),
                positions=torch.tensor([2, 3, 4], **i32), slots=torch.tensor([18, 19, 20], device="cuda"),
                page_list=torch.tensor([[1]], **i32), kv_lens=torch.tensor([5], **i32),
                q_starts=torch.tensor([0, 3], **i32))


def rope(a):
    return paged.qk_norm_rope(a["q"], a["k"], a["positions"], a["table"], a["q_weight"], a["k_weight"])


def append(a):
    paged.kv_append(a["k"], a["v"], a["k_cache"], a["v_cache"], a["slots"], a["positions"], a["table"], a["k_weight"])


def attend(a):
    return paged.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["page_list"], a["kv_lens"], a["q_starts"], 3, 5)


@pytest.mark.parametrize("call,names", [
    (rope, ("q", "k", "q_weight", "k_weight")), (append, ("k", "v", "k_cache", "v_cache", "k_weight")),
    (attend, ("q", "k_cache", "v_cache"))])
def test_gradients_are_not_dropped_silently(call, names):
    for name in names:
        a = arguments()
        a[name] = a[name].detach().requires_grad_()
        with pytest.raises(ft.FtcnnError, match="no backward"):
            call(a)
            pytest.fail(f"{name} that requires a gradient was not refused")
        with torch.no_grad():
            call(a)
        with torch.inference_mode():
            call(a)
        a[name] = a[name].detach()
        call(a)


def test_keys_alone_and_queries_alone_that_require_gradients():
    a = arguments()
    k = a["k"].detach().requires_grad_()
    for q, k in ((None, k), (k, None)):
        with pytest.raises(ft.FtcnnError, match="no backward"):
            paged.qk_norm_rope(q, k)


def test_heads_of_no_values():
    a = arguments()
    for name in ("q", "k_cache", "v_cache"):
        a[name] = a[name][..., :0]
    with pytest.raises(ft.FtcnnError, match="dim 0"):
        attend(a)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices in one process")
def test_every_device_of_the_process():
    """Kernels whose LDS is more than a launch has unasked, on one device after the other."""
    outs = []
    for i in range(torch.cuda.device_count()):
        with torch.cuda.device(i):
            torch.manual_seed(1)
            q = torch.randn(40, 4, 256).to("cuda")
            cache = torch.randn(2, 4, 16, 2, 256).to("cuda")
            i32 = dict(dtype=torch.int32, device="cuda")
            outs.append(paged.paged_attention(q, cache[0], cache[1], torch.arange(4, **i32).view(1, 4),
                                              torch.tensor([60], **i32), torch.tensor([0, 40], **i32), 40, 60).cpu())
    assert all(torch.equal(o, outs[0]) for o in outs) and torch.isfinite(outs[0]).all()


def test_without_torch_s_short_ways_to_stream_and_device(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.delattr(torch._C, "_cuda_getDevice")
    spec = importlib.util.spec_from_file_location("paper_2003_12203_amd.paged_again", paged.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    monkeypatch.undo()
    a = arguments()
    append(a)
    args = (a["q"], a["k_cache"], a["v_cache"], a["page_list"], a["kv_lens"], a["q_starts"], 3, 5)
    assert torch.equal(again.paged_attention(*args), attend(a))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = again.paged_attention(*args, stream=s)
    s.synchronize()
    assert torch.equal(got, attend(a))
