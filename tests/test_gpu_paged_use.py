"""The serving operators as a program uses them: on a stream of their own, captured in a graph, called again
with the same bits, refused with what does not fit, and together in a layer (examples/attention_layer.py)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2003_12203_amd as ft
from oracle import serving as sv
from paper_2003_12203_amd import paged

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def example():
    spec = importlib.util.spec_from_file_location("attention_layer", os.path.join(ROOT, "examples", "attention_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def f64(t):
    return t.detach().cpu().double().numpy()


def step(seed, dtype, new, length, heads=8, kv=2, dim=64, page=16):
    """Everything that a layer's step takes, on the device; the cache holds the tokens before."""
    rng = np.random.default_rng(seed)
    count = [-(-n // page) for n in length]
    pages = sum(count) + 1
    lists = np.zeros((len(new), max(count)), np.int32)
    free, at = rng.permutation(pages), 0
    for b, n in enumerate(count):
        lists[b, :n] = free[at:at + n]
        at += n
    seq = np.concatenate([np.full(n, b) for b, n in enumerate(new)])
    pos = np.concatenate([np.arange(l - n, l) for n, l in zip(new, length)])
    cache = paged.PagedCache(pages, page, kv, dim, dtype)
    for c in (cache.k, cache.v):
        c.copy_(torch.from_numpy(rng.standard_normal(c.shape)).to(c.dtype))
    s = dict(
        cache=cache, qkv=torch.from_numpy(rng.standard_normal((sum(new), heads + 2 * kv, dim))).to("cuda", DT[dtype]),
        positions=torch.from_numpy(pos.astype(np.int32)).cuda(), page_list=torch.from_numpy(lists).cuda(),
        kv_lens=torch.tensor(length, dtype=torch.int32, device="cuda"),
        q_starts=torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32, device="cuda"),
        table=paged.rope_table(max(length) + 8, dim), weight=torch.rand(dim, device="cuda") + 0.5,
        heads=heads, kv=kv, max_q=max(new), max_kv=max(length))
    s["slots"] = cache.slots(s["page_list"], torch.from_numpy(seq).cuda(), s["positions"])
    return s


def run(s, out=None, stream=None, lse=None, workspace=None):
    h, kv, qkv, cache = s["heads"], s["kv"], s["qkv"], s["cache"]
    q, _ = paged.qk_norm_rope(qkv[:, :h], None, s["positions"], s["table"], s["weight"], stream=stream)
    paged.kv_append(qkv[:, h:h + kv], qkv[:, h + kv:], cache.k, cache.v, s["slots"], s["positions"], s["table"],
                    s["weight"], stream=stream)
    return paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], s["max_q"],
                                 s["max_kv"], out=out, lse=lse, workspace=workspace, stream=stream)


STEPS = [([1] * 5, [300, 17, 1, 4000, 64]),       # single tokens, split
         ([130, 1, 40], [130, 900, 70]),           # a prompt, a token, a chunk
         ([200], [6000])]                          # a chunk over many keys, split


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,length", STEPS)
def test_the_same_bits_again(dtype, new, length):
    s = step(1, dtype, new, length)
    first = run(s)
    for _ in range(4):
        torch.randn(1 << 20, device="cuda").sort()   # other work in between
        assert torch.equal(run(s), first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,length", STEPS)
def test_steps_in_a_graph(dtype, new, length):
    """A captured step replays with what its tensors then hold: other tokens, other lengths, other pages."""
    s, others = step(2, dtype, new, length), [step(3 + i, dtype, new, length) for i in range(3)]
    out = torch.empty_like(s["qkv"][:, :s["heads"]], memory_format=torch.contiguous_format)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(s, out)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(s, out)
    for i, o in enumerate(others * 2):
        o["kv_lens"].sub_(1 if i >= 3 else 0).clamp_(min=1)   # shorter the second time
        want = run(o)
        for name in ("qkv", "positions", "page_list", "kv_lens", "q_starts", "slots", "weight"):
            s[name].copy_(o[name])
        s["cache"].k.copy_(o["cache"].k)
        s["cache"].v.copy_(o["cache"].v)
        torch.cuda.synchronize()
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(s["cache"].k, o["cache"].k) and torch.equal(s["cache"].v, o["cache"].v)


def test_on_a_stream_of_its_own():
    """All three on a stream that is not the current one, in order with what that stream did before."""
    s = step(9, "bf16", [40, 1], [700, 3000])
    want = run(s)
    qkv = s["qkv"].clone()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s["qkv"].zero_()
        torch.randn(1 << 22, device="cuda").sort()
        s["qkv"].copy_(qkv)
    got = run(s, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)


def test_a_given_workspace_and_one_that_does_not_fit():
    s = step(10, "bf16", [1], [20000])
    want = run(s)
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    assert torch.equal(run(s, workspace=room), want)
    room.fill_(255)                                   # what it holds does not matter
    assert torch.equal(run(s, workspace=room), want)
    with pytest.raises(ft.FtcnnError, match="workspace"):
        run(s, workspace=room[:100])
    with pytest.raises(ft.FtcnnError, match="256-byte"):
        run(s, workspace=room[16:])


def test_out_may_be_q():
    for new, length in STEPS:
        s = step(11, "bf16", new, length)
        q = s["qkv"][:, :s["heads"]].contiguous()
        args = (s["cache"].k, s["cache"].v, s["page_list"], s["kv_lens"], s["q_starts"], s["max_q"], s["max_kv"])
        want = paged.paged_attention(q, *args)
        assert torch.equal(paged.paged_attention(q, *args, out=q), want)


def test_the_binding_refuses():
    s = step(12, "bf16", [3], [40])
    h, kv, qkv, cache = s["heads"], s["kv"], s["qkv"], s["cache"]
    q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
    pos, table, w = s["positions"], s["table"], s["weight"]
    bad = [
        lambda: paged.qk_norm_rope(q.half(), None), lambda: paged.qk_norm_rope(q[0], None),
        lambda: paged.qk_norm_rope(q, k[:2]), lambda: paged.qk_norm_rope(q, k.float()),
        lambda: paged.qk_norm_rope(q, None, pos), lambda: paged.qk_norm_rope(q, None, None, table),
        lambda: paged.qk_norm_rope(q, None, pos.long(), table), lambda: paged.qk_norm_rope(q, None, pos[:2], table),
        lambda: paged.qk_norm_rope(q, None, pos.cpu(), table), lambda: paged.qk_norm_rope(q, None, pos, table.bfloat16()),
        lambda: paged.qk_norm_rope(q, None, pos, table[..., 0]), lambda: paged.qk_norm_rope(q, None, pos, table, w[:8]),
        lambda: paged.qk_norm_rope(q, None, pos, table, w.half()), lambda: paged.qk_norm_rope(q, k, pos, table, w, w.bfloat16()),
        lambda: paged.qk_norm_rope(q, None, pos, table, layout="other"), lambda: paged.qk_norm_rope(q, None, q_out=k),
        lambda: paged.qk_norm_rope(q.transpose(0, 2).contiguous().transpose(0, 2), None),
        lambda: paged.kv_append(k, v[:, :1], cache.k, cache.v, s["slots"]),
        lambda: paged.kv_append(k, v.float(), cache.k, cache.v, s["slots"]),
        lambda: paged.kv_append(k, v, cache.k[:, :, :1], cache.v, s["slots"]),
        lambda: paged.kv_append(k, v, cache.k, cache.v[:1], s["slots"]),
        lambda: paged.kv_append(k, v, cache.k, cache.v, s["slots"].int()),
        lambda: paged.kv_append(k, v, cache.k, cache.v, s["slots"][:2]),
        lambda: paged.paged_attention(q, cache.k.float(), cache.v, s["page_list"], s["kv_lens"], s["q_starts"]),
        lambda: paged.paged_attention(q, cache.k, cache.v[:1], s["page_list"], s["kv_lens"], s["q_starts"]),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"].long(), s["kv_lens"], s["q_starts"]),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"].long(), s["q_starts"]),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"][:1]),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"]),   # three tokens of one
        lambda: paged.paged_attention(q[:, :3], cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"]),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], scale=-1.0),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], window=-1),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], window=4,
                                      causal=False),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], lse=w),
        lambda: paged.paged_attention(q, cache.k, cache.v, s["page_list"], s["kv_lens"], s["q_starts"], out=k),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ft.FtcnnError):
            call()
            pytest.fail(f"call {i} was not refused")
    run(s)   # and what fits still runs
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_step_by_step(dtype):
    """The example's layer: each operator within its bound of the definitions, on what the one before it
    made; a fault planted in either projection is corrected."""
    ex = example()
    hidden, heads, kv, dim, page = 256, 8, 2, 64, 16
    cache = paged.PagedCache(24, page, kv, dim, dtype)
    layer = ex.AttentionLayer(hidden, heads, kv, dim, cache, 256, dtype)
    seqs = ex.Sequences(3, 24, page, 10)
    table, w = f64(layer.table), f64(layer.k_weight)
    rng = torch.Generator().manual_seed(5)
    for new in ([50, 7, 0], [33, 1, 20], [1, 1, 1], [1, 0, 1]):
        st = seqs.step(new)
        before = f64(cache.k), f64(cache.v)
        x = torch.randn(sum(new), hidden, generator=rng).to("cuda", DT[dtype])
        fault = dict(n=x.shape[0] - 1, m=3, x=0, y=0, kind="set", value=1e6)
        y = layer(x, st, ((fault,), (fault,)))
        assert [l.read_report().status for l in layer.reports] == [ft.STATUS_CORRECTED] * 2
        assert y.shape == x.shape and torch.isfinite(y).all()
        qkv, pos = f64(layer.qkv), st["positions"].cpu().numpy()
        want, bound = sv.norm_rope(qkv[:, :heads], pos, table, f64(layer.q_weight), dtype=dtype)
        assert (np.abs(f64(layer.q) - want) <= bound).all()
        slots = cache.slots(st["page_list"], st["seq"], st["positions"]).cpu().numpy()
        kn, kb = sv.norm_rope(qkv[:, heads:heads + kv], pos, table, w, dtype=dtype)
        wk, wv = sv.append(*before, kn, qkv[:, heads + kv:], slots)
        bk, _ = sv.append(np.zeros_like(before[0]), before[1], kb, kb, slots)
        assert (np.abs(f64(cache.k) - wk) <= bk).all() and np.array_equal(f64(cache.v), wv)
        out, _, bo, _ = sv.attention(f64(layer.q), f64(cache.k), f64(cache.v), st["page_list"].cpu().numpy(),
                                     st["kv_lens"].cpu().numpy(), st["q_starts"].cpu().numpy(), dtype=dtype)
        assert (np.abs(f64(layer.attended) - out) <= bo).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_example(dtype):
    """Prompts in chunks and single tokens through the whole layer against float64.  Rounding: in bf16, queries and
    keys of unit size are off by 2^-8 each, a score (a sum of 64 such products, scaled) by about 2^-7, outputs by
    a few percent, their largest of some 10^5 by four times that; in fp32, 2^-16 of these.  A page, position or head mistaken
    is off by more than one."""
    worst, corrected = example().serve(dtype, new=5)
    assert worst < (0.5 if dtype == "bf16" else 1e-3)
    assert corrected >= 8   # one a step: three steps of prompts, five of single tokens and more


@pytest.mark.parametrize("dtype,dim,rot,layout", [
    ("bf16", 128, 128, "half"), ("bf16", 128, 24, "half"), ("bf16", 72, 72, "interleaved"), ("bf16", 96, 90, "half"),
    ("f32", 128, 64, "interleaved"), ("f32", 80, 32, "half"), ("f32", 60, 20, "half")])
def test_norms_and_rotation_of_many_tokens(dtype, dim, rot, layout):
    """Several heads to a lane group and outputs past the L2s, in vectors of every width."""
    rng = np.random.default_rng([dim, rot])
    tokens, heads, kv = 1201, 120, 24
    qkv = torch.from_numpy(rng.standard_normal((tokens, heads + kv, dim)).astype(np.float32)).to("cuda", DT[dtype])
    pos = torch.from_numpy(rng.permutation(tokens).astype(np.int32)).cuda()
    table, w = paged.rope_table(tokens, rot), torch.from_numpy(rng.random((2, dim)).astype(np.float32) + 0.5).cuda()
    q, k = paged.qk_norm_rope(qkv[:, :heads], qkv[:, heads:], pos, table, w[0], w[1], layout=layout)
    for got, x, weight in ((q, qkv[:, :heads], w[0]), (k, qkv[:, heads:], w[1])):
        want, bound = sv.norm_rope(f64(x), pos.cpu().numpy(), f64(table), f64(weight), layout=layout, dtype=dtype)
        assert (np.abs(f64(got) - want) <= bound).all()


def test_numbers_that_do_not_fit_are_refused():
    s = step(13, "f32", [1], [20])
    q = s["qkv"][:, :s["heads"]]
    args = (q, s["cache"].k, s["cache"].v, s["page_list"], s["kv_lens"])
    with pytest.raises(ft.FtcnnError, match="does not hold"):
        paged.paged_attention(*args, max_kv=1 << 40)
    with pytest.raises(ft.FtcnnError, match="does not hold"):
        paged.paged_attention(*args, scale=1e300)
    with pytest.raises(ft.FtcnnError, match="does not hold"):
        paged.qk_norm_rope(q, None, eps=1e300)


@pytest.mark.parametrize("new", [1, 9])
def test_more_sequences_than_lanes(new):
    """The schedule over 150 ragged sequences, some of them empty, and the cut units among them."""
    rng = np.random.default_rng(new)
    length = [int(n) for n in rng.integers(new, 700, 150)]
    length[3] = length[64] = length[149] = 0
    length[70] = 6000
    news = [min(new, n) if b % 7 else 0 for b, n in enumerate(length)]
    news[70] = new
    s = step(14, "bf16", news, length, heads=4, kv=2)
    out = run(s)
    lse = torch.empty(sum(news), 4, device="cuda")
    run(s, lse=lse)
    h = s["heads"]
    q, _ = paged.qk_norm_rope(s["qkv"][:, :h], None, s["positions"], s["table"], s["weight"])
    want, wl, bo, bl = sv.attention(f64(q), f64(s["cache"].k), f64(s["cache"].v), s["page_list"].cpu().numpy(), length,
                                    s["q_starts"].cpu().numpy(), dtype="bf16")
    assert (np.abs(f64(out) - want) <= bo).all()
    assert (np.abs(f64(lse) - wl) <= bl).all()
