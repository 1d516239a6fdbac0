"""The operators of a serving attention layer from their definitions, numpy float64: norms and rotation,
the paged cache, attention.  Each result comes with the bound that fp32 arithmetic (and the stated
rounding of softmax weights) keeps to, element by element.

Sums of n terms in fp32 in any order are within n 2^-24 of their sum of magnitudes; a product, a
rounding or a call of exp2, log2 or rsqrt within 2^-23 (one unit in the last place) of its value.
"""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # half a unit in the last place of 24 and 8 bits


def rope_table(max_pos, rot, base=10000.0, scaling="plain", factor=1.0, original=0, low=1.0, high=32.0, amplitude=1.0):
    """[max_pos][rot / 2][2]: cos and sin of p * f_j."""
    out = np.zeros((max_pos, rot // 2, 2))
    for j in range(rot // 2):
        b = base
        if scaling == "base" and rot > 2:
            b = base * factor ** (rot / (rot - 2.0))
        f = b ** (-2.0 * j / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            turns = original * f / (2.0 * np.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = f * keep + f / factor * (1.0 - keep)
        angle = np.arange(max_pos) * f
        out[:, j, 0], out[:, j, 1] = np.cos(angle) * amplitude, np.sin(angle) * amplitude
    return out


def pairs(rot, layout):
    """The indices of each pair's two values."""
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def norm_rope(x, positions=None, table=None, weight=None, eps=1e-6, layout="half", dtype="f32"):
    """x [tokens][heads][dim] -> (y, bound)."""
    x = np.asarray(x, np.float64)
    dim = x.shape[-1]
    y, rel = x.copy(), 0.0
    if weight is not None:
        y = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * np.asarray(weight, np.float64)
        # the mean square within dim units, its root half of that; then the root, two products
        rel = (dim / 2 + 8) * U32
    mag = np.abs(y)
    if positions is not None:
        z, size = y.copy(), mag.copy()
        a, b = pairs(2 * table.shape[1], layout)
        for t, p in enumerate(positions):
            if not 0 <= p < table.shape[0]:
                z[t][:, a] = z[t][:, b] = np.nan
                continue
            c, s = table[p, :, 0].astype(np.float64), table[p, :, 1].astype(np.float64)
            z[t][:, a] = y[t][:, a] * c - y[t][:, b] * s
            z[t][:, b] = y[t][:, b] * c + y[t][:, a] * s
            size[t][:, a] = mag[t][:, a] * np.abs(c) + mag[t][:, b] * np.abs(s)
            size[t][:, b] = mag[t][:, b] * np.abs(c) + mag[t][:, a] * np.abs(s)
        y, mag, rel = z, size, rel + 4 * U32
    copied = weight is None and positions is None
    bound = rel * mag + (0.0 if copied else U_OUT[dtype]) * (np.abs(y) + rel * mag)
    return y, bound


def append(k_cache, v_cache, k, v, slots):
    """Copies of the caches [pages][page][heads][dim] with the tokens' rows in them."""
    kc, vc = k_cache.copy(), v_cache.copy()
    pages, page = kc.shape[:2]
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            kc[s // page, s % page], vc[s // page, s % page] = k[t], v[t]
    return kc, vc


def attention(q, k_cache, v_cache, page_list, kv_lens, q_starts=None, scale=None, causal=True, window=0, dtype="f32"):
    """-> (out, lse, bound of out, bound of lse); tokens of no sequence are 0, their lse -inf."""
    q = np.asarray(q, np.float64)
    tokens, heads, dim = q.shape
    page, kv_heads = k_cache.shape[1:3]
    group = heads // kv_heads
    scale = 1.0 / np.sqrt(dim) if scale is None else scale
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    bo, bl = np.zeros(q.shape), np.zeros(q.shape[:2])
    u_p = U_OUT["bf16"] if dtype == "bf16" else U32   # the weights as the product takes them
    for b, n in enumerate(kv_lens):
        n = int(n)
        lo, hi = (b, b + 1) if q_starts is None else (int(q_starts[b]), int(q_starts[b + 1]))
        rows = [(int(page_list[b][j // page]), j % page) for j in range(n)]
        for h in range(kv_heads):
            K = np.array([k_cache[r][h] for r in rows], np.float64).reshape(n, dim)
            V = np.array([v_cache[r][h] for r in rows], np.float64).reshape(n, dim)
            for t in range(lo, hi):
                p = n - (hi - lo) + (t - lo)
                first = max(0, p - window + 1) if window else 0
                last = min(p, n - 1) if causal else n - 1
                for g in range(h * group, (h + 1) * group):
                    if last < first:
                        out[t, g], lse[t, g] = 0.0, -np.inf
                        continue
                    k, v = K[first:last + 1], V[first:last + 1]
                    s = k @ q[t, g] * scale
                    top = s.max()
                    e = np.exp(s - top)
                    w = e / e.sum()
                    with np.errstate(invalid="ignore"):
                        out[t, g] = w @ v
                        size = w @ np.abs(v)
                    lse[t, g] = top + np.log(e.sum())
                    # a score is within ds; a weight, relative, within ds (its own) + ds (the sum's);
                    # two sums of n terms, the weights' rounding, exp2 and its argument, a few products
                    with np.errstate(invalid="ignore"):
                        ds = (dim + 8) * U32 * scale * (np.abs(k) @ np.abs(q[t, g])).max() + 8 * U32 * np.abs(s).max()
                    rel = 2 * ds + u_p + 2 * (len(s) + 32) * U32
                    bo[t, g] = rel * size + U_OUT[dtype] * np.abs(out[t, g]) * (1 + rel)
                    bl[t, g] = ds + (len(s) + 32) * U32 + 4 * U32 * abs(lse[t, g])
    return out, lse, bo, bl


def low_rank_add(y, x, a, b, ids, scales=None, ranks=None, dtype="f32"):
    """-> (out, bound): y[t] + scales[i] b[i] (a[i] x[t]) of the first ranks[i] rows of a[i], i = ids[t].

    A value of a x is within (ch + 8) units of its sum of magnitudes (ch terms in any order, the scale's product among
    the rest); as two bf16 values within 2^-16 of itself; the sum over the rank within (rank + 4) units of its own."""
    y, x, a, b = (np.asarray(t, np.float64) for t in (y, x, a, b))
    out, bound = y.copy(), np.zeros(y.shape)
    for t, i in enumerate(ids):
        if not 0 <= i < a.shape[0]:
            continue
        r = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        s = 1.0 if scales is None else float(scales[i])
        low, size = s * (a[i, :r] @ x[t]), abs(s) * (np.abs(a[i, :r]) @ np.abs(x[t]))
        off = (x.shape[1] + 8) * U32 * size + (2.0 ** -16 * np.abs(low) if dtype == "bf16" else 0.0)
        add, mag = b[i, :, :r] @ low, np.abs(b[i, :, :r]) @ np.abs(low)
        err = np.abs(b[i, :, :r]) @ off
        err = err + (r + 4) * U32 * (mag + err)
        out[t] = y[t] + add
        bound[t] = err + (U32 + U_OUT[dtype]) * (np.abs(out[t]) + err)
    return out, bound


def attention_mass(mass, q, k_cache, page_list, kv_lens, lse, q_starts=None, scale=None, causal=True, window=0):
    """-> (mass, bound): to mass[b][j] the weights exp(s - lse) of the rows and heads that see position j."""
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    heads, dim = q.shape[1:]
    page, kv_heads = k_cache.shape[1:3]
    group = heads // kv_heads
    scale = 1.0 / np.sqrt(dim) if scale is None else scale
    out = np.array(mass, np.float64)
    bound = np.zeros(out.shape)
    for b, n in enumerate(kv_lens):
        n = int(n)
        lo, hi = (b, b + 1) if q_starts is None else (int(q_starts[b]), int(q_starts[b + 1]))
        rows = [(int(page_list[b][j // page]), j % page) for j in range(n)]
        add, err, terms = np.zeros(n), np.zeros(n), np.zeros(n)
        for h in range(kv_heads):
            K = np.array([k_cache[r][h] for r in rows], np.float64).reshape(n, dim)
            for t in range(lo, hi):
                p = n - (hi - lo) + (t - lo)
                first = max(0, p - window + 1) if window else 0
                last = min(p, n - 1) if causal else n - 1
                if last < first:
                    continue
                seen = slice(first, last + 1)
                for g in range(h * group, (h + 1) * group):
                    s = K[seen] @ q[t, g] * scale
                    w = np.exp(s - lse[t, g])
                    # a score's sum and products; the argument's two roundings and the power's
                    ds = (dim + 8) * U32 * scale * (np.abs(K[seen]) @ np.abs(q[t, g])) + 8 * U32 * np.abs(s)
                    ds = ds + 4 * U32 * (np.abs(lse[t, g]) + np.abs(s - lse[t, g]) + 1)
                    add[seen] += w
                    err[seen] += w * np.expm1(ds) + 2.0 ** -120
                    terms[seen] += 1
        out[b, :n] += add
        bound[b, :n] = err + (terms + 8) * U32 * (add + err) + 2 * U32 * np.abs(out[b, :n])
    return out, bound


def evict(k_cache, v_cache, page_list, kv_lens, keep, mass, positions=None, first=0, since=None):
    """-> (k_cache, v_cache, lens, mass, positions), exactly."""
    kc, vc = k_cache.copy(), v_cache.copy()
    page = kc.shape[1]
    lens, out, pos = [], np.zeros(mass.shape, np.float32), np.full(mass.shape, -1, np.int32)
    for b, n in enumerate(kv_lens):
        n = int(n)
        k = min(max(int(keep[b]), 0), n)
        p = [int(x) for x in positions[b][:n]] if positions is not None else list(range(n))
        late = int(since[b]) if since is not None else 1 << 40

        def order(j):
            w = float(mass[b][j])
            return (not (p[j] < first or p[j] >= late), w != w, 0.0 if w != w else -w, j)

        stay = set(sorted(range(n), key=order)[:k])
        holes, movers = [j for j in range(k) if j not in stay], [j for j in range(k, n) if j in stay]
        source = list(range(k))
        for to, at in zip(holes, movers):
            source[to] = at
            rt, ra = (int(page_list[b][to // page]), to % page), (int(page_list[b][at // page]), at % page)
            kc[rt], vc[rt] = kc[ra], vc[ra]
        out[b, :k], pos[b, :k] = mass[b][source], [p[j] for j in source]
        lens.append(k)
    return kc, vc, np.array(lens, np.int32), out, pos
