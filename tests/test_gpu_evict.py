"""Eviction from a paged cache (ftcnn_evict) against its definition: every value and index exactly."""
import numpy as np
import pytest
import torch

import paper_2003_12203_amd as ft
from oracle import serving as sv
from paper_2003_12203_amd import paged

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(seed, length, keep, kv=2, dim=16, page=16, dtype="bf16", order="heads", kind="heavy", positions=False, extra=1):
    rng = np.random.default_rng(seed)
    count = [-(-n // page) for n in length]
    pages = sum(count) + 2
    free, at = rng.permutation(pages), 0
    lists = np.full((len(length), max(count) + extra), 10 ** 9, np.int32)
    for b, n in enumerate(count):
        lists[b, :n] = free[at:at + n]
        at += n
    shape = (pages, kv, page, dim) if order == "heads" else (pages, page, kv, dim)
    k, v = (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda", DT[dtype]) for _ in range(2))
    if order == "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    places = lists.shape[1] * page
    mass = np.exp(2 * rng.standard_normal((len(length), places))).astype(np.float32)
    if kind == "ties":
        mass = rng.integers(0, 3, mass.shape).astype(np.float32)
    elif kind == "equal":
        mass[:] = 0.25
    elif kind == "odd":
        some = np.array([0.0, -0.0, np.nan, -np.nan, np.inf, -np.inf, 1e-45, -1e-45, 1.0, -1.0, 3e38], np.float32)
        mass = rng.choice(some, mass.shape)
    elif kind == "near":   # differ in their last bits only
        mass = (np.float32(1.0).view(np.int32) + rng.integers(0, 40, mass.shape)).astype(np.int32).view(np.float32)
    pos = None
    if positions:
        pos = torch.from_numpy(np.argsort(np.argsort(rng.random(mass.shape), 1), 1).astype(np.int32)).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(k=k, v=v, lists=torch.from_numpy(lists).cuda(), lens=torch.tensor(length, **i32), keep=torch.tensor(keep, **i32),
                mass=torch.from_numpy(mass).cuda(), positions=pos)


def run(s, **kw):
    return paged.evict(s["k"], s["v"], s["lists"], s["lens"], s["keep"], s["mass"], s["positions"], **kw)


def host(t):
    return None if t is None else t.detach().cpu().float().numpy() if t.is_floating_point() else t.cpu().numpy()


def check(s, first=0, since=None, **kw):
    """Runs the call on s and compares all it leaves; returns what it returned."""
    want = sv.evict(host(s["k"]), host(s["v"]), host(s["lists"]), host(s["lens"]), host(s["keep"]), host(s["mass"]),
                    host(s["positions"]), first, host(since))
    lens, mass, positions = run(s, first=first, since=since, **kw)
    places = s["lists"].shape[1] * s["k"].shape[1]
    assert np.array_equal(host(lens), want[2])
    for got, w, name in ((s["k"], want[0], "keys"), (s["v"], want[1], "values"), (mass[:, :places], want[3][:, :places], "mass"),
                         (positions[:, :places], want[4][:, :places], "positions")):
        got = host(got)
        same = np.array_equal(got.view(np.int32) if got.dtype == np.float32 else got, w.view(np.int32) if w.dtype == np.float32 else w)
        assert same, name
    return lens, mass, positions


LENGTHS = [([1], [0]), ([1], [1]), ([2], [1]), ([5, 0, 3], [2, 4, 3]), ([64], [63]), ([65, 63], [1, 62]), ([1000, 17, 1024], [500, 17, 1]),
           ([1025, 2049], [1024, 700]), ([300, 299, 298], [-4, 10 ** 9, 150])]


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "odd", "near"])
@pytest.mark.parametrize("i", range(len(LENGTHS)))
def test_exactly(i, kind):
    s = make(i, *LENGTHS[i], kind=kind, dtype="f32" if i % 2 else "bf16", page=(16, 24, 5)[i % 3], order=("heads", "rows")[i % 2])
    check(s)


@pytest.mark.parametrize("kind", ["heavy", "ties", "odd"])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("first,recent", [(0, 0), (4, 0), (0, 40), (5, 30), (400, 400), (10 ** 6, 0)])
def test_positions_that_are_kept(first, recent, positions, kind):
    """Some, all that stay, and more than may stay."""
    s = make(first + recent, [600, 33, 0, 257], [200, 32, 5, 256], kind=kind, positions=positions)
    since = (s["lens"] - recent).int() if recent else None
    check(s, first, since)


@pytest.mark.parametrize("n,k", [(16384, 9000), (16385, 1), (16448, 16447), (40000, 20011), (70001, 333)])
@pytest.mark.parametrize("kind", ["heavy", "ties"])
def test_long_sequences(n, k, kind):
    """About what a workgroup holds in registers, and past it."""
    s = make(n, [n, 50], [k, 20], kv=1, dim=8, page=64, kind=kind, positions=True)
    check(s, 3, torch.tensor([n - 100, 45], dtype=torch.int32, device="cuda"), max_kv=n)


LONG = [20000, 0, 16384, 40000, 9, 33000, 32768, 17000]


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "odd", "near"])
@pytest.mark.parametrize("first,recent", [(0, 0), (3, 90), (0, 38000)])
def test_long_and_short_together(first, recent, kind):
    """Sequences of several parts beside shorter ones; all, some or none of what stays is kept for its position."""
    s = make(12, LONG, [16385, 4, 16383, 30000, 3, 33000, 1, 0], kv=1, dim=8, page=48, kind=kind, positions=recent == 90)
    check(s, first, (s["lens"] - recent).int() if recent else None)


def test_long_in_place_and_graph():
    spec = dict(length=[40000, 20000], keep=[9000, 19990], kv=1, dim=8, page=64, positions=True)
    t = make(13, **spec)
    graph = torch.cuda.CUDAGraph()
    held = dict(lens_out=t["lens"], mass_out=t["mass"], positions_out=t["positions"])
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")   # (larger than the call asks for)
    with torch.cuda.graph(graph):
        run(t, first=2, workspace=room, **held)
    for seed in range(3):
        new = make(40 + seed, **spec)
        for k in ("k", "v", "lists", "lens", "keep", "mass", "positions"):
            t[k].copy_(new[k])
        graph.replay()
        want = check(new, 2)
        assert all(torch.equal(a, b) for a, b in zip((t["lens"], t["mass"], t["positions"]), want))
        assert torch.equal(new["k"], t["k"]) and torch.equal(new["v"], t["v"])


@pytest.mark.parametrize("kv,dim,dtype", [(1, 8, "bf16"), (1, 8, "f32"), (3, 72, "bf16"), (8, 128, "bf16"), (12, 256, "f32"), (40, 40, "bf16")])
def test_rows_of_any_size(kv, dim, dtype):
    for order in ("heads", "rows"):
        check(make(kv * dim, [150, 90], [70, 60], kv=kv, dim=dim, dtype=dtype, order=order))


def test_in_place_and_hints():
    for hint in (0, 1, 100, 10 ** 6):
        s, t = (make(7, [500, 40, 300], [220, 40, 299], positions=True) for _ in range(2))
        want = check(s, 2)
        got = run(t, first=2, max_kv=hint, lens_out=t["lens"], mass_out=t["mass"], positions_out=t["positions"])
        assert got[0] is t["lens"] and got[1] is t["mass"] and got[2] is t["positions"]
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        assert torch.equal(s["k"], t["k"]) and torch.equal(s["v"], t["v"])


@pytest.mark.parametrize("n,hint", [(5000, 1), (5000, 1025), (40000, 100), (17000, 16384), (9000, 40000)])
def test_hints_that_are_wrong(n, hint):
    """Longer sequences than the caller said, and lists for far more than there is."""
    s = make(n, [n, 70], [n // 3, 69], kv=1, dim=8, page=64, kind="ties", positions=True, extra=300)
    check(s, 3, torch.tensor([n - 100, 60], dtype=torch.int32, device="cuda"), max_kv=hint)


def test_layouts():
    """Caches inside larger ones, a mass and positions with rows of their own and more places than the lists name."""
    s = make(8, [200, 100], [90, 99], kv=2, dim=32, page=16, positions=True)
    pages = s["k"].shape[0]
    wide = torch.full((pages, 16, 2, 2, 48), 3.0, dtype=torch.bfloat16, device="cuda")
    k, v = wide[:, :, 0, :, 8:40], wide[:, :, 1, :, 16:]
    k.copy_(s["k"]), v.copy_(s["v"])
    places = s["mass"].shape[1]
    mass, pos = torch.full((2, places + 50), 9.0, device="cuda"), torch.full((2, places + 30), 9, dtype=torch.int32, device="cuda")
    mass[:, 5:5 + places], pos[:, 3:3 + places] = s["mass"], s["positions"]
    t = dict(s, k=k, v=v, mass=mass[:, 5:-1], positions=pos[:, 3:-1])
    mass_out, pos_out = torch.full((2, places + 9), 8.0, device="cuda"), torch.full((2, places + 9), 8, dtype=torch.int32, device="cuda")
    want = check(s, 4)
    got = run(t, first=4, mass_out=mass_out[:, 2:], positions_out=pos_out[:, 4:])
    assert torch.equal(k, s["k"]) and torch.equal(v, s["v"]) and torch.equal(got[0], want[0])
    assert torch.equal(mass_out[:, 2:2 + places], want[1]) and torch.equal(pos_out[:, 4:4 + places], want[2])
    for t, a, b in ((mass_out, 2, 7), (pos_out, 4, 5)):
        assert (t[:, :a] == 8).all() and (t[:, a + places:] == 8).all()
    assert (wide[:, :, 0, :, :8] == 3).all() and (wide[:, :, 0, :, 40:] == 3).all() and (wide[:, :, 1, :, :16] == 3).all()


def test_what_index_arrays_say_is_brought_into_range():
    s = make(9, [40, 30], [20, 12])
    s["lens"] = torch.tensor([10 ** 9, -3], dtype=torch.int32, device="cuda")
    s["lists"][0, 2:] = torch.tensor([-5, 10 ** 9], dtype=torch.int32, device="cuda")[:s["lists"].shape[1] - 2]
    lens, mass, positions = run(s)
    assert lens.tolist() == [20, 0] and mass[1].eq(0).all() and positions[1].eq(-1).all()
    assert mass[0, :20].gt(0).all() and mass[0, 20:].eq(0).all()


def test_no_sequences_and_no_pages():
    s = make(10, [4], [2])
    empty = run(dict(s, lists=s["lists"][:0], lens=s["lens"][:0], keep=s["keep"][:0], mass=s["mass"][:0]))
    assert [tuple(t.shape) for t in empty] == [(0,), (0, 32), (0, 32)]
    lens, mass, positions = run(dict(s, lists=s["lists"][:, :0], mass=s["mass"][:, :0]))
    assert lens.tolist() == [0] and mass.shape == positions.shape == (1, 0)


def test_same_bits_streams_and_graphs():
    spec = dict(length=[900, 64, 333], keep=[400, 63, 5], positions=True)
    s, t = make(11, **spec), make(11, **spec)
    want = run(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(t, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(s["k"], t["k"]) and torch.equal(s["v"], t["v"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run(t)
    for seed in range(3):
        new = make(30 + seed, **spec)
        for k in ("k", "v", "lists", "lens", "keep", "mass", "positions"):
            t[k].copy_(new[k])
        graph.replay()
        eager = run(new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)) and torch.equal(new["k"], t["k"]) and torch.equal(new["v"], t["v"])


def test_cache_past_32_bits():
    s = make(12, [60, 40], [25, 30])
    far, pages = (1 << 29) - 8, s["k"].shape[0]
    rooms = [torch.empty(far * (pages - 1) + 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = (r.as_strided(s["k"].shape, (far, 16, 256, 1)) for r in rooms)
    k.copy_(s["k"]), v.copy_(s["v"])
    run(dict(s, k=k, v=v))
    check(s)
    assert torch.equal(k, s["k"]) and torch.equal(v, s["v"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_cache_kept_at_its_budget(dtype):
    """As a program uses it: single tokens appended, attended, weighed and evicted, step after step, beside a float64
    account of which rows each sequence holds and what weight they got."""
    rng = np.random.default_rng(13)
    heads, kv, dim, page, budget, batch = 4, 2, 32, 8, 21, 3
    cache = paged.PagedCache(batch * 4, page, kv, dim, dtype)
    lists = torch.from_numpy(rng.permutation(batch * 4).reshape(batch, 4).astype(np.int32)).cuda()
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    keep = torch.tensor([budget, budget - 4, 50], dtype=torch.int32, device="cuda")
    mass, positions = torch.zeros(batch, 32, device="cuda"), torch.full((batch, 32), -1, dtype=torch.int32, device="cuda")
    held = [dict() for _ in range(batch)]   # position -> (key, value, weight)
    seq = torch.arange(batch, device="cuda")
    for step in range(30):
        q, k, v = (torch.from_numpy(rng.standard_normal((batch, h, dim)).astype(np.float32)).to("cuda", DT[dtype]) for h in (heads, kv, kv))
        paged.kv_append(k, v, cache.k, cache.v, cache.slots(lists, seq, lens))
        positions[seq, lens.long()] = step
        lens += 1
        lse = torch.empty(batch, heads, device="cuda")
        out = paged.paged_attention(q, cache.k, cache.v, lists, lens, lse=lse)
        paged.attention_mass(mass, q, cache.k, lists, lens, lse)
        since = torch.full((batch,), step - 4, dtype=torch.int32, device="cuda")
        weights = mass.cpu()
        at = positions.cpu()
        paged.evict(cache.k, cache.v, lists, lens, keep, mass, positions, 2, since, lens_out=lens, mass_out=mass, positions_out=positions)
        for b in range(batch):
            held[b][step] = (k[b].cpu().double(), v[b].cpu().double(), 0.0)
            ps = sorted(held[b])
            K, V = (torch.stack([held[b][p][i] for p in ps]).repeat_interleave(heads // kv, 1) for i in (0, 1))
            w = torch.softmax(torch.einsum("hd,phd->hp", q[b].cpu().double(), K) * dim ** -0.5, -1)
            want = torch.einsum("hp,phd->hd", w, V)
            assert (out[b].cpu().double() - want).abs().max() <= (2 ** -8 if dtype == "bf16" else 2 ** -18) * V.abs().max()
            for p, x in zip(ps, w.sum(0).tolist()):
                held[b][p] = held[b][p][:2] + (held[b][p][2] + x,)
            n = len(ps)
            place = {int(at[b, j]): j for j in range(n)}
            assert sorted(place) == ps
            for p in ps:   # at most 30 steps of 4 weights, each within a few units of 32 terms
                assert abs(float(weights[b, place[p]]) - held[b][p][2]) <= 2 ** -15 * (1 + held[b][p][2])
            k_now = min(int(keep[b]), n)
            order = sorted(ps, key=lambda p: (not (p < 2 or p >= step - 4), -float(weights[b, place[p]]), place[p]))
            held[b] = {p: held[b][p] for p in order[:k_now]}
            assert int(lens[b]) == k_now and sorted(positions[b, :k_now].tolist()) == sorted(held[b])
            assert mass[b, k_now:].eq(0).all() and positions[b, k_now:].eq(-1).all()


def test_binding_refuses():
    s = make(14, [40, 30], [20, 12], positions=True)
    args = dict(k_cache=s["k"], v_cache=s["v"], page_list=s["lists"], kv_lens=s["lens"], keep=s["keep"], mass=s["mass"],
                positions=s["positions"])
    bad = [("k_cache", s["k"].half()), ("k_cache", s["k"].cpu()), ("v_cache", s["v"].float()), ("v_cache", s["v"][:, :8]),
           ("page_list", s["lists"].long()), ("kv_lens", s["lens"][:1]), ("keep", s["keep"].long()), ("keep", s["keep"][:1]),
           ("mass", s["mass"][:, :-1]), ("mass", s["mass"].double()), ("positions", s["positions"].long()),
           ("positions", s["positions"][:, :-1])]
    for k, v in bad:
        with pytest.raises(ft.FtcnnError, match="evict"):
            paged.evict(**{**args, k: v})
    for kw in (dict(first=-1), dict(max_kv=-1), dict(since=s["lens"].float()), dict(lens_out=s["lens"][:1]),
               dict(mass_out=s["mass"][:1].expand(2, -1)), dict(positions_out=s["mass"]), dict(first=2 ** 40),
               dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ft.FtcnnError, match="evict"):
            paged.evict(**args, **kw)
    with pytest.raises(ft.FtcnnError, match="no backward"):
        paged.evict(**{**args, "mass": s["mass"].clone().requires_grad_()})


@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("given", ["none", "mass", "other"])
def test_allocated_positions_have_the_lists_places(given, positions):
    """Whatever the width of the weights that are given and of the positions that are read: a place for every row that the lists can
    name, and each of them written."""
    s = make(15, [200, 0, 70], [90, 5, 69], positions=True)
    places = s["mass"].shape[1]
    wide = {k: torch.nn.functional.pad(s[k], (0, 33), value=5) for k in ("mass", "positions")}
    t = dict(s, k=s["k"].clone(), v=s["v"].clone(), mass=wide["mass"], positions=wide["positions"] if positions else None)
    want = check(s if positions else dict(s, positions=None), 4)
    mass_out = {"none": None, "mass": t["mass"], "other": torch.full_like(wide["mass"], 7.0)}[given]
    lens, mass, pos = run(t, first=4, mass_out=mass_out)
    assert pos.shape == (3, places) and pos.dtype == torch.int32
    assert torch.equal(pos, want[2]) and torch.equal(mass[:, :places], want[1]) and torch.equal(lens, want[0])
    assert mass.shape == ((3, places) if given == "none" else wide["mass"].shape)
    assert given == "none" or (mass[:, places:] == (5 if given == "mass" else 7)).all()   # what is not the lists' is left


def test_weights_and_positions_of_overlapping_rows():
    """Windows of one array, a place apart or the same for all, are read like any others, and what is allocated has rows of its own."""
    s = make(16, [60, 64, 33], [20, 63, 30], extra=0)
    places = s["mass"].shape[1]
    base = torch.rand(places + 2, generator=torch.Generator().manual_seed(1)).cuda()
    for mass, pos in ((base.unfold(0, places, 1), torch.arange(5, places + 7, dtype=torch.int32, device="cuda").unfold(0, places, 1)),
                      (base[:places].expand(3, -1), torch.arange(places, dtype=torch.int32, device="cuda").expand(3, -1))):
        assert mass.stride(0) < 2 and pos.stride(0) < 2
        for positions in (pos, None):
            t = dict(s, k=s["k"].clone(), v=s["v"].clone(), mass=mass, positions=positions)
            want = check(dict(t, k=t["k"].clone(), v=t["v"].clone(), mass=mass.contiguous(),
                              positions=None if positions is None else positions.contiguous()), 6)
            got = check(t, 6)
            assert all(torch.equal(a, b) and a.is_contiguous() for a, b in zip(got, want))


@pytest.mark.parametrize("moves", [6143, 6144, 6145, 8192])
@pytest.mark.parametrize("kind", ["rising", "recent"])
@pytest.mark.parametrize("positions", [False, True])
def test_every_row_that_stays_moves(moves, kind, positions):
    """16384 places, as many as a workgroup keeps in LDS, of which the last stay, for their weights or their positions: as many
    moves as lists in LDS hold, one less and more, and the most that there are; in place as well."""
    n = 16384

    def fresh():
        s = make(moves, [n, 30], [moves, 29], kv=1, dim=8, page=64, extra=0)
        if kind == "rising":
            s["mass"] = torch.arange(n, dtype=torch.float32, device="cuda").expand(2, n).contiguous()
        if positions:
            s["positions"] = torch.arange(n, dtype=torch.int32, device="cuda").expand(2, n).contiguous()
        return s

    s, t = fresh(), fresh()
    since = torch.tensor([n - moves, 10], dtype=torch.int32, device="cuda") if kind == "recent" else None
    want = check(s, 0, since, max_kv=n)
    assert want[2][0, :moves].tolist() == list(range(n - moves, n))
    held = dict(lens_out=t["lens"], mass_out=t["mass"])
    if positions:
        held["positions_out"] = t["positions"]
    got = run(t, since=since, max_kv=n, **held)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert torch.equal(s["k"], t["k"]) and torch.equal(s["v"], t["v"])
