"""The attention weight that cached keys get (ftcnn_attention_mass) against its definition in float64."""
import numpy as np
import pytest
import torch

import paper_2003_12203_amd as ft
from oracle import serving as sv
from paper_2003_12203_amd import paged

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().cpu().double().numpy()


def make(seed, dtype, new, length, heads, kv, dim, page, order="heads", spare=2):
    """Sequences of new[b] new and length[b] cached tokens, the lse that their attention gives, some mass before."""
    rng = np.random.default_rng(seed)
    count = [-(-n // page) for n in length]
    pages = sum(count) + spare
    free = rng.permutation(pages)
    lists = np.full((len(new), max(1, max(count)) + 1), -7, np.int32)   # past a sequence: any number
    at = 0
    for b, n in enumerate(count):
        lists[b, :n] = free[at:at + n]
        at += n
    shape = (pages, kv, page, dim) if order == "heads" else (pages, page, kv, dim)
    cache = [torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda", DT[dtype]) for _ in range(2)]
    if order == "heads":
        cache = [c.transpose(1, 2) for c in cache]
    q = torch.from_numpy(rng.standard_normal((sum(new), heads, dim)).astype(np.float32)).to("cuda", DT[dtype])
    return dict(q=q, k=cache[0], v=cache[1], lists=torch.from_numpy(lists).cuda(),
                lens=torch.tensor(length, dtype=torch.int32, device="cuda"),
                starts=torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32, device="cuda"),
                mass=torch.from_numpy(rng.random((len(new), lists.shape[1] * page)).astype(np.float32)).cuda())


def with_lse(s, **kw):
    s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    paged.paged_attention(s["q"], s["k"], s["v"], s["lists"], s["lens"], s["starts"], lse=s["lse"], **kw)
    return s


def call(s, mass=None, starts=True, **kw):
    mass = s["mass"].clone() if mass is None else mass
    return paged.attention_mass(mass, s["q"], s["k"], s["lists"], s["lens"], s["lse"], s["starts"] if starts else None, **kw)


def check(s, got, causal=True, window=0, scale=None):
    want, bound = sv.attention_mass(f64(s["mass"]), f64(s["q"]), f64(s["k"]), s["lists"].cpu().numpy(), s["lens"].tolist(),
                                    f64(s["lse"]), s["starts"].tolist(), scale, causal, window)
    got = f64(got)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    off = np.abs(got - want)[~nan] - bound[~nan]
    assert off.max() <= 0, f"{(off > 0).sum()} of {off.size} over, by {off.max()}"
    for b, n in enumerate(s["lens"].tolist()):
        assert torch.equal(torch.from_numpy(got[b, n:]).float(), s["mass"][b, n:].cpu())   # past the rows: as it was


CASES = [  # new, length, heads, kv, dim, page, window, causal
    ([1], [1], 1, 1, 8, 1, 0, True), ([1], [77], 8, 2, 128, 16, 0, True), ([1, 1, 1], [5, 0, 130], 4, 4, 64, 24, 0, True),
    ([1, 1], [300, 129], 10, 5, 72, 16, 0, True), ([1, 1], [140, 33], 16, 1, 256, 5, 40, True),
    ([4, 1, 3], [260, 1, 64], 4, 1, 96, 16, 0, True), ([5, 0, 2], [5, 9, 1], 6, 3, 40, 7, 0, True),
    ([17, 40], [300, 40], 4, 2, 128, 16, 0, True), ([130], [130], 8, 2, 64, 64, 0, True),
    ([70, 3, 0], [500, 260, 10], 6, 2, 80, 24, 33, True), ([65], [270], 5, 1, 256, 16, 0, False),
    ([33, 64], [64, 20], 4, 4, 136, 3, 0, True), ([200], [200], 2, 1, 192, 200, 70, True), ([3, 2], [150, 140], 2, 1, 64, 16, 0, False),
    ([129, 1], [700, 513], 2, 2, 8, 16, 1, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_float64(i, dtype):
    new, length, heads, kv, dim, page, window, causal = CASES[i]
    s = make(i, dtype, new, length, heads, kv, dim, page, "heads" if i % 2 else "rows")
    with_lse(s, causal=causal, window=window)
    check(s, call(s, causal=causal, window=window, max_q=max(new), max_kv=max(length)), causal, window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [1, 2, 3, 4, 8, 12, 32, 64, 80])
@pytest.mark.parametrize("window,causal", [(0, True), (250, True), (0, False)])
def test_tiles_of_tokens_heads(group, window, causal, dtype):
    """Tokens' heads together in tiles, or one head's rows; last tiles that are not full, before keys that all rows see."""
    new, length = [33, 3, 129, 64, 17], [600, 700, 900, 520, 16]
    s = make(group, dtype, new, length, group, 1, 64, 16)
    with_lse(s, causal=causal, window=window)
    check(s, call(s, causal=causal, window=window, max_q=129, max_kv=900), causal, window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_last_rows_that_are_not_finite(dtype):
    """The last token's queries, which stand in for the rows behind it, reach only the keys that it sees."""
    s = make(63, dtype, [49, 40], [400, 300], 8, 2, 128, 16)
    s["q"][48, 3, 5], s["q"][88, 7, 0] = float("nan"), float("inf")
    with_lse(s)
    got = call(s, max_q=49, max_kv=400)
    assert got[0, :400].isnan().all() and torch.equal(got[0, 400:], s["mass"][0, 400:])
    clean = dict(s, q=s["q"].clone())
    clean["q"][88, 7, 0] = clean["q"][48, 3, 5] = 1.0
    with_lse(clean)
    assert got[1, 299].isnan() and not call(clean, max_q=49, max_kv=400).isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_hints_shape_the_launch_only(dtype):
    """Too small, too large or missing: another order of the sums, and both kernels over any count of rows."""
    s = make(50, dtype, [40, 1, 9], [400, 290, 9], 4, 2, 64, 16)
    with_lse(s)
    for hints in ((0, 0), (1, 1), (1, 4000), (4000, 1), (40, 400), (3, 100)):
        check(s, call(s, max_q=hints[0], max_kv=hints[1]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [40, 72, 200])
@pytest.mark.parametrize("window,causal", [(0, True), (50, True), (0, False)])
def test_lists_for_far_more_than_is_cached(dim, window, causal, dtype):
    """Launches shaped for many keys: 64 of them to a wave, parts of many workgroups."""
    new, length = [70, 1, 130, 64], [300, 90, 130, 700]
    s = make(62, dtype, new, length, 4, 2, dim, 16)
    with_lse(s, causal=causal, window=window)
    wide = torch.full((4, 2000), -1, dtype=torch.int32, device="cuda")
    wide[:, :s["lists"].shape[1]] = s["lists"]
    s["lists"], s["mass"] = wide, torch.rand(4, 2000 * 16, device="cuda")
    check(s, call(s, causal=causal, window=window), causal, window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,most", [(70, 1), (130, 1), (200, 1), (70, 40)])
def test_many_sequences(batch, most, dtype):
    """More than a wave's lanes, many of them empty or without new tokens."""
    rng = np.random.default_rng(batch)
    new = rng.integers(1 if most == 1 else 0, most + 1, batch)
    length = new * (rng.random(batch) < 0.7) * 1 + rng.integers(0, 2, batch) * rng.integers(0, 90, batch)
    s = with_lse(make(63, dtype, new.tolist(), length.tolist(), 4, 2, 16, 8))
    check(s, call(s, max_q=most, max_kv=int(length.max())))


def test_single_tokens_need_no_starts():
    s = with_lse(make(51, "bf16", [1, 1, 1], [30, 200, 0], 8, 2, 128, 16))
    assert torch.equal(call(s, starts=False), call(s, max_q=1))


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_of_a_row_add_to_one(dtype, many):
    s = with_lse(make(52, dtype, [37 if many else 1], [900], 8, 2, 128, 16))
    got = call(s, torch.zeros_like(s["mass"]))
    assert abs(float(got.double().sum()) / (8 * (37 if many else 1)) - 1) < 1e-5   # 900 terms of 2^-21 each, far apart


@pytest.mark.parametrize("new", [[1, 1], [30, 20]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_nobody_sees(new, dtype):
    """NaN and infinities in rows past a sequence, in keys that causal rows do not see, and in other pages."""
    s = with_lse(make(53, dtype, new, [75, 61], 4, 2, 64, 16))
    clean = call(s)
    used = set()
    for b, n in enumerate(s["lens"].tolist()):
        page = int(s["lists"][b, (n - 1) // 16])
        s["k"][page, (n - 1) % 16 + 1:] = float("nan")
        used |= set(s["lists"][b, :(n - 1) // 16 + 1].tolist())
    for page in set(range(s["k"].shape[0])) - used:
        s["k"][page] = float("inf")
    assert torch.equal(call(s), clean)
    if new[0] > 1:   # the last token's key: only that token sees it
        page, row = int(s["lists"][0, 74 // 16]), 74 % 16
        s["k"][page, row] = float("nan")
        got = call(s)
        assert got[0, 74].isnan() and torch.equal(got[0, :74], clean[0, :74]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("new", [1, 40])
def test_a_row_that_is_not_finite(new):
    s = with_lse(make(54, "bf16", [new, 1], [80, 50], 4, 2, 64, 16))
    clean = call(s)
    s["q"][0, 1, 3] = float("nan")
    got = call(s)
    seen = 80 - new + 1
    assert got[0, :seen].isnan().all() and torch.equal(got[0, seen:], clean[0, seen:]) and torch.equal(got[1], clean[1])


def test_rows_that_see_nothing():
    """More new tokens than cached ones, an empty cache: their lse is -infinity, and they add nothing."""
    s = with_lse(make(55, "bf16", [6, 2, 20], [4, 0, 3], 4, 2, 64, 16))
    assert s["lse"][:2].eq(-float("inf")).all()
    check(s, call(s))


@pytest.mark.parametrize("new", [[1, 1], [20, 20]])
def test_what_index_arrays_say_is_brought_into_range(new):
    s = with_lse(make(56, "bf16", new, [40, 30], 4, 2, 64, 16))
    clean = call(s)
    odd = dict(s)
    odd["lens"] = torch.tensor([40, -5], dtype=torch.int32, device="cuda")
    got = call(odd)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], s["mass"][1])
    odd = dict(s, lists=s["lists"].clone(), lens=torch.tensor([10 ** 9, 30], dtype=torch.int32, device="cuda"))
    odd["lists"][0, 1:] = torch.tensor([10 ** 9, -10 ** 9, 5], dtype=torch.int32, device="cuda")[:odd["lists"].shape[1] - 1]
    got = call(odd)
    assert torch.equal(got[1], clean[1]) and got[0].isfinite().all()
    odd = dict(s, starts=torch.tensor([-4, new[0], 10 ** 9], dtype=torch.int32, device="cuda"))
    assert torch.equal(call(odd)[0], clean[0])


@pytest.mark.parametrize("new", [[1, 1], [50, 30]])
def test_padding_around_the_sequences(new):
    """Rows before q_starts[0] and behind the last belong to nobody, whatever they hold."""
    s = with_lse(make(57, "bf16", new, [70, 60], 4, 2, 64, 16))
    clean = call(s, max_q=max(new))
    pad = torch.full((3, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    s["q"] = torch.cat((pad, s["q"], pad))
    s["lse"] = torch.cat((torch.full((3, 4), float("nan"), device="cuda"), s["lse"], torch.full((3, 4), float("nan"), device="cuda")))
    s["starts"] = s["starts"] + 3
    assert torch.equal(call(s, max_q=max(new)), clean)


@pytest.mark.parametrize("new", [[1, 1, 1], [30, 60, 5]])
def test_layouts(new):
    """Queries inside packed rows, a mass with rows of its own, more places than the lists name."""
    s = with_lse(make(58, "bf16", new, [90, 70, 20], 4, 2, 64, 16))
    want = call(s)
    packed = torch.zeros(sum(new), 8, 72, dtype=torch.bfloat16, device="cuda")
    q = packed[:, 2:6, 8:]
    q.copy_(s["q"])
    room = torch.full((3, 300), 5.0, device="cuda")
    mass = room[:, 11:11 + s["mass"].shape[1] + 4]
    mass[:, :s["mass"].shape[1]] = s["mass"]
    got = call(dict(s, q=q), mass)
    assert got is mass and torch.equal(mass[:, :want.shape[1]], want)
    assert (room[:, :11] == 5).all() and (room[:, 11 + want.shape[1]:] == 5).all()


@pytest.mark.parametrize("new,length", [([1] * 4, [700, 10, 300, 0]), ([90, 20], [600, 300]), ([257], [257])])
def test_same_bits_streams_and_graphs(new, length):
    s = with_lse(make(59, "bf16", new, length, 8, 2, 128, 16))
    want = call(s, max_q=max(new), max_kv=max(length))
    assert torch.equal(call(s, max_q=max(new), max_kv=max(length)), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mass = s["mass"].clone()
    side.wait_stream(torch.cuda.current_stream())
    call(s, mass, stream=side, max_q=max(new), max_kv=max(length))
    side.synchronize()
    assert torch.equal(mass, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, mass, max_q=max(new), max_kv=max(length))
    for seed in range(3):
        other = with_lse(make(70 + seed, "bf16", new, length, 8, 2, 128, 16))
        for k in ("q", "k", "lists", "lse"):
            s[k].copy_(other[k])
        mass.copy_(other["mass"])
        graph.replay()
        graph.replay()   # it adds
        eager = call(other, max_q=max(new), max_kv=max(length))
        call(other, eager, max_q=max(new), max_kv=max(length))
        torch.cuda.synchronize()
        assert torch.equal(mass, eager)


def test_cache_past_32_bits():
    """Pages that lie more than 2^31 values from the first."""
    s = with_lse(make(60, "bf16", [1, 20], [40, 50], 4, 2, 64, 16))
    want = call(s)
    pages = s["k"].shape[0]
    far = (1 << 29) - 8
    room = torch.empty(far * (pages - 1) + 16 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    k = room.as_strided(s["k"].shape, (far, 64, 16 * 64, 1))
    k.copy_(s["k"])
    assert torch.equal(call(dict(s, k=k)), want)


def test_binding_refuses():
    s = with_lse(make(61, "bf16", [1, 1], [20, 30], 4, 2, 64, 16))
    args = dict(mass=s["mass"], q=s["q"], k_cache=s["k"], page_list=s["lists"], kv_lens=s["lens"], lse=s["lse"])
    bad = [("mass", s["mass"].double()), ("mass", s["mass"][:, :-1]), ("mass", s["mass"][:1]), ("mass", s["mass"].cpu()),
           ("mass", s["mass"][:1].expand(2, -1)), ("q", s["q"].half()), ("q", s["q"][:, :3]), ("k_cache", s["k"].float()),
           ("k_cache", s["k"][..., :56]), ("page_list", s["lists"].long()), ("kv_lens", s["lens"][:1]), ("lse", s["lse"][:1]),
           ("lse", s["lse"].double()), ("q", s["q"].cpu())]
    for k, v in bad:
        with pytest.raises(ft.FtcnnError, match="attention_mass"):
            paged.attention_mass(**{**args, k: v})
    for kw in (dict(q_starts=s["starts"][:2]), dict(window=-1), dict(window=3, causal=False), dict(scale=0.0),
               dict(scale=float("nan")), dict(max_kv=-1), dict(max_kv=2 ** 40)):
        with pytest.raises(ft.FtcnnError, match="attention_mass"):
            paged.attention_mass(**args, **kw)
    with pytest.raises(ft.FtcnnError, match="no backward"):
        paged.attention_mass(**{**args, "q": s["q"].clone().requires_grad_()})
