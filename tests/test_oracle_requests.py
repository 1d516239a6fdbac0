"""oracle.serving's adapters, attention mass and eviction against torch's own float64 operations and by hand, and
mistakes planted in them that their bounds have to show (CPU)."""
import numpy as np
import pytest
import torch

from oracle import serving as sv
from test_oracle_serving import problem


def adapted(seed, tokens=9, ch=40, m=24, count=3, rank=8):
    rng = np.random.default_rng(seed)
    ids = rng.integers(-1, count, tokens)
    return (rng.standard_normal((tokens, m)), rng.standard_normal((tokens, ch)), rng.standard_normal((count, rank, ch)),
            rng.standard_normal((count, m, rank)), ids, rng.random(count) + 0.5, rng.integers(0, rank + 3, count))


def dense_adapted(y, x, a, b, ids, scales, ranks):
    out = torch.from_numpy(y).clone()
    for t, i in enumerate(ids):
        if i >= 0:
            w = torch.from_numpy(b[i][:, :ranks[i]]) @ torch.from_numpy(a[i][:ranks[i]])   # the adapter as one matrix
            out[t] += scales[i] * (w @ torch.from_numpy(x[t]))
    return out.numpy()


@pytest.mark.parametrize("seed", range(4))
def test_low_rank_add(seed):
    args = adapted(seed)
    out, bound = sv.low_rank_add(*args)
    assert np.allclose(out, dense_adapted(*args), rtol=0, atol=1e-11)
    none = args[4] < 0
    assert np.array_equal(out[none], args[0][none]) and (bound[none] == 0).all() and bound.max() < 1e-2
    fp32 = [x.astype(np.float32) if x.dtype == np.float64 else x for x in args]   # plain fp32 keeps to the bound
    exact, bound = sv.low_rank_add(*fp32)
    got = fp32[0].copy()
    for t, i in enumerate(args[4]):
        if i >= 0:
            r = min(args[6][i], 8)
            got[t] += fp32[3][i][:, :r] @ (fp32[5][i] * (fp32[2][i][:r] @ fp32[1][t]))
    assert (np.abs(got - exact) <= bound).all()


@pytest.mark.parametrize("mistake", ["scale", "rank", "adapter", "channel"])
def test_low_rank_add_shows_mistakes(mistake):
    y, x, a, b, ids, scales, ranks = adapted(7)
    ids[:3], ranks[:] = [0, 1, 2], [8, 5, 3]
    want, bound = sv.low_rank_add(y, x, a, b, ids, scales, ranks, dtype="bf16")
    if mistake == "scale":
        scales = scales * 1.01
    elif mistake == "rank":
        ranks = ranks - 1
    elif mistake == "adapter":
        ids = np.roll(ids, 1)
    else:
        x = np.where(np.arange(x.shape[1]) == 39, 0, x)
    got, _ = sv.low_rank_add(y, x, a, b, ids, scales, ranks, dtype="bf16")
    assert (np.abs(got - want) > 2 * bound).any()


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 6), (False, 0)])
@pytest.mark.parametrize("new,length", [([1], [1]), ([3, 1], [9, 30]), ([5, 0, 2], [5, 7, 0]), ([6], [4]), ([20], [33])])
def test_attention_mass(new, length, causal, window):
    q, kc, vc, lists, lens, starts = problem(sum(new), new, length)
    _, lse, _, _ = sv.attention(q, kc, vc, lists, lens, starts, causal=causal, window=window)
    before = np.random.default_rng(0).random((len(new), lists.shape[1] * 4))
    got, bound = sv.attention_mass(before, q, kc, lists, lens, lse, starts, causal=causal, window=window)
    # the same as the weights on values that are one at a key's place
    one = np.zeros((kc.shape[0], 4, 2, 64))
    for b, n in enumerate(length):
        for j in range(n):
            one[lists[b][j // 4], j % 4, :, j] = 1.0
    for b, n in enumerate(length):
        lo, hi = starts[b], starts[b + 1]
        w = np.zeros(64)
        if hi > lo and n:
            wide = np.concatenate((q[lo:hi], np.zeros((hi - lo, 4, 48))), -1)
            keys = np.concatenate((kc, np.zeros((*kc.shape[:3], 48))), -1)
            out, *_ = sv.attention(wide, keys, one, lists[b:b + 1], [n], [0, hi - lo], scale=0.25, causal=causal, window=window)
            w = out.sum((0, 1))
        assert np.allclose(got[b, :n] - before[b, :n], w[:n], rtol=0, atol=1e-12)
        assert np.array_equal(got[b, n:], before[b, n:])
    assert (bound >= 0).all() and bound.max() < 1e-4


@pytest.mark.parametrize("mistake", ["causal", "window", "scale", "head"])
def test_attention_mass_shows_mistakes(mistake):
    q, kc, vc, lists, lens, starts = problem(3, [5, 2], [30, 21])
    kw = dict(causal=True, window=9)
    _, lse, _, _ = sv.attention(q, kc, vc, lists, lens, starts, **kw)
    zero = np.zeros((2, lists.shape[1] * 4))
    want, bound = sv.attention_mass(zero, q, kc, lists, lens, lse, starts, **kw)
    if mistake == "causal":
        starts = [0, 4, 7]
    elif mistake == "window":
        kw["window"] = 8
    elif mistake == "scale":
        kw["scale"] = 0.2501
    else:
        q = q[:, [1, 0, 2, 3]]
    got, _ = sv.attention_mass(zero, q, kc, lists, lens, lse, starts, **kw)
    assert (np.abs(got - want) > 2 * bound).any()


def test_evict_by_hand():
    """Nine rows in pages of four; five stay: 0 (first), 8 (late), and the heaviest of the rest, of equal ones the lower."""
    k = np.arange(3 * 4, dtype=np.float32).reshape(3, 4, 1, 1)
    mass = np.array([[0, 5, 1, 3, 3, 3, np.nan, 4, 0, 7, 7, 7]], np.float32)
    kc, vc, lens, out, pos = sv.evict(k, k + 100, [[2, 0, 1]], [9], [5], mass, None, 1, [8])
    # 0, 1, 3, 7, 8 stay; place 2 takes row 7, place 4 row 8
    assert lens.tolist() == [5] and pos[0].tolist() == [0, 1, 7, 3, 8] + [-1] * 7
    assert out[0].tolist() == [0, 5, 4, 3, 0] + [0] * 7
    rows = kc[[2, 0, 1]].reshape(-1)
    assert rows[:5].tolist() == [8, 9, 3, 11, 4] and (vc[[2, 0, 1]].reshape(-1)[:5] == rows[:5] + 100).all()
    assert rows[5:].tolist() == [1, 2, 3, 4, 5, 6, 7]   # the rest as it was


def test_evict_orders_odd_weights():
    mass = np.array([[np.nan, -np.inf, -0.0, 0.0, np.inf, -1.0, 1e-45, np.nan]], np.float32)
    k = np.zeros((2, 4, 1, 1), np.float32)
    stays = [set(sv.evict(k, k, [[0, 1]], [8], [n], mass)[4][0][:n].tolist()) for n in range(9)]
    order = [min(stays[n + 1] - stays[n]) for n in range(8)]
    assert order == [4, 6, 2, 3, 5, 1, 0, 7]
    many = sv.evict(k, k, [[0, 1]], [8], [3], np.arange(8, dtype=np.float32)[None], None, 6)   # more kept than may stay
    assert set(many[4][0][:3].tolist()) == {3, 4, 5}
