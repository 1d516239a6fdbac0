"""oracle.serving against torch's own float64 operations and by hand, and mistakes planted in it that its
bounds have to show (CPU)."""
import numpy as np
import pytest
import torch

from oracle import serving as sv


def problem(seed, new, length, heads=4, kv=2, dim=16, page=4):
    rng = np.random.default_rng(seed)
    count = [-(-n // page) for n in length]
    lists = np.full((len(new), max(max(count), 1)), -1)
    free = rng.permutation(sum(count) + 1)
    at = 0
    for b, n in enumerate(count):
        lists[b, :n] = free[at:at + n]
        at += n
    cache = rng.standard_normal((2, sum(count) + 1, page, kv, dim))
    q = rng.standard_normal((sum(new), heads, dim))
    return q, cache[0], cache[1], lists, length, np.concatenate(([0], np.cumsum(new)))


def dense(q, kc, vc, lists, lens, starts, causal=True, window=0):
    """The same with torch.softmax over gathered rows."""
    heads, dim = q.shape[1:]
    page, kv = kc.shape[1:3]
    out, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full(q.shape[:2], -torch.inf, dtype=torch.float64)
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        if n == 0 or hi == lo:
            continue
        k = torch.from_numpy(kc[lists[b]].reshape(-1, kv, dim)[:n]).repeat_interleave(heads // kv, 1)
        v = torch.from_numpy(vc[lists[b]].reshape(-1, kv, dim)[:n]).repeat_interleave(heads // kv, 1)
        s = torch.einsum("thd,jhd->htj", torch.from_numpy(q[lo:hi]), k) / dim ** 0.5
        p, j = torch.arange(n - (hi - lo), n)[:, None], torch.arange(n)[None]
        see = (j <= p) if causal else torch.ones(hi - lo, n, dtype=torch.bool)
        if window:
            see = see & (j > p - window)
        s = s.masked_fill(~see, -torch.inf)
        out[lo:hi] = torch.einsum("htj,jhd->thd", torch.softmax(s, -1).nan_to_num(0.0), v)
        lse[lo:hi] = torch.logsumexp(s, -1).T
    return out.numpy(), lse.numpy()


CASES = [([1], [1]), ([3, 1], [9, 30]), ([5, 0, 2], [5, 7, 0]), ([6], [4]), ([20], [33])]


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 6), (False, 0)])
@pytest.mark.parametrize("new,length", CASES)
def test_attention(new, length, causal, window):
    args = problem(len(length) * 10 + sum(new), new, length)
    out, lse, bo, bl = sv.attention(*args, causal=causal, window=window)
    want = dense(*args, causal=causal, window=window)
    assert np.allclose(out, want[0], rtol=0, atol=1e-13)
    assert np.array_equal(np.isinf(lse), np.isinf(want[1]))
    ok = np.isfinite(lse)
    assert np.allclose(lse[ok], want[1][ok], rtol=0, atol=1e-13)
    assert (bo >= 0).all() and (bl >= 0).all() and bo.max() < 1e-3


def test_attention_by_hand():
    # two keys, the second twice as likely as the first
    q, kc = np.ones((1, 1, 1)), np.zeros((1, 2, 1, 1))
    kc[0, 1] = np.log(2.0)
    vc = np.array([3.0, 6.0]).reshape(1, 2, 1, 1)
    out, lse, _, _ = sv.attention(q, kc, vc, [[0]], [2], scale=1.0)
    assert np.isclose(out[0, 0, 0], 5.0) and np.isclose(lse[0, 0], np.log(3.0))


@pytest.mark.parametrize("mistake", ["a key too many", "a page swapped", "another head", "no scale"])
def test_mistakes_in_the_attention_are_beyond_its_bounds(mistake):
    q, kc, vc, lists, lens, starts = problem(5, [2, 3], [9, 14])
    out, _, bo, _ = sv.attention(q, kc, vc, lists, lens, starts, dtype="bf16")
    kw = {}
    if mistake == "a key too many":
        kw["causal"] = False
    elif mistake == "a page swapped":
        lists = lists.copy()
        lists[1, [0, 2]] = lists[1, [2, 0]]
        lists[1, 0], lists[1, 1] = lists[1, 1], lists[0, 0]
    elif mistake == "another head":
        kc, vc = kc[:, :, ::-1], vc[:, :, ::-1]
    else:
        kw["scale"] = 1.0
    wrong = sv.attention(q, kc, vc, lists, lens, starts, **kw)[0]
    assert (np.abs(wrong - out) > bo).any()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(8, 8), (12, 4), (2, 2)])
def test_rotation_is_a_complex_product(layout, dim, rot):
    rng = np.random.default_rng(dim)
    x, pos = rng.standard_normal((5, 3, dim)), np.array([0, 1, 7, 30, 99])
    table = sv.rope_table(100, rot)
    y, bound = sv.norm_rope(x, pos, table, layout=layout)
    a, b = sv.pairs(rot, layout)
    turn = np.exp(1j * pos[:, None] * 10000.0 ** (-2.0 * np.arange(rot // 2) / rot))[:, None]
    z = (x[..., a] + 1j * x[..., b]) * turn
    assert np.allclose(y[..., a], z.real, rtol=0, atol=1e-13) and np.allclose(y[..., b], z.imag, rtol=0, atol=1e-13)
    assert np.array_equal(y[..., rot:], x[..., rot:])
    assert np.array_equal(y[0], x[0])   # position 0 turns nothing
    # scores of rotated rows depend on the positions' distance alone
    same = np.broadcast_to(x[:1], x.shape)
    one = sv.norm_rope(same, np.array([3, 10, 20, 40, 90]), table, layout=layout)[0]
    two = sv.norm_rope(same[:, ::-1], np.array([5, 12, 22, 42, 92]), table, layout=layout)[0]
    s = (one * two).sum(-1)
    assert np.allclose(s, s[:1], rtol=0, atol=1e-12)
    assert (np.abs(sv.norm_rope(x, pos + 1 - 2 * (pos > 50), table, layout=layout)[0] - y) > bound).any()


def test_norm():
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((4, 2, 10)), rng.standard_normal(10)
    y, _ = sv.norm_rope(x, weight=w, eps=1e-3)
    t = torch.from_numpy(x)
    want = torch.nn.functional.rms_norm(t, (10,), torch.from_numpy(w), 1e-3).numpy()
    assert np.allclose(y, want, rtol=0, atol=1e-13)


def test_table_scalings():
    plain = sv.rope_table(50, 32)
    assert np.allclose(sv.rope_table(50, 32, scaling="linear", factor=2.0)[::2], plain[:25], rtol=0, atol=1e-12)
    based = sv.rope_table(50, 32, scaling="base", factor=4.0)
    assert np.allclose(based[:, 0], plain[:, 0], rtol=0, atol=1e-12)                # the fastest pair is kept
    assert np.allclose(based[::4, -1], plain[:13, -1], rtol=0, atol=1e-12)          # the slowest slowed by factor
    parts = sv.rope_table(50, 32, scaling="parts", factor=4.0, original=40, low=1.0, high=4.0)
    assert np.allclose(parts[:, 0], plain[:, 0], rtol=0, atol=1e-12)                # 6.4 turns: kept
    assert np.allclose(parts[::4, -1], plain[:13, -1], rtol=0, atol=1e-12)          # less than one turn: slowed


def test_append():
    rng = np.random.default_rng(4)
    kc, vc = rng.standard_normal((2, 3, 4, 1, 2))
    k, v = rng.standard_normal((2, 3, 1, 2))
    a, b = sv.append(kc, vc, k, v, [5, -1, 12])
    assert np.array_equal(a[1, 1], k[0]) and np.array_equal(b[1, 1], v[0])
    a[1, 1], b[1, 1] = kc[1, 1], vc[1, 1]
    assert np.array_equal(a, kc) and np.array_equal(b, vc)
