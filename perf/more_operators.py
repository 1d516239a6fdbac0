"""The operators of a batch whose requests differ, as cases to time and to check.

Requests that one attention layer serves together bring their own low-rank adapters beside the shared
projections, and keep their caches within their own budgets:

``low_rank_add``    each token's adapter, added to the output of a projection that all tokens share
``attention_mass``  the softmax weight that every cached key got from the new tokens, summed
``evict``           the rows with the least of it taken out of each sequence's pages

Where ``own`` is false, ``run`` computes them with elementary torch operations in 32 bits; where it
is true, it makes the calls of ``paper_2003_12203_amd.adapters`` and ``paper_2003_12203_amd.paged``.
``exact`` has them in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# the most that a drawn case takes: that of the largest listed ones
MAX_FLOPS = 5.6e11        # attention_mass, in products
MAX_SCORES = 4.2e9        # ... and in the scores of its plain form
MAX_CACHE = 1.4e8         # values of all cached keys
MAX_ADAPT = 5.2e10        # low_rank_add, in the products of its plain form
MAX_ROWS = 1.01e8         # ... and in the values of its rows


def _adapt(name, tokens, ch, m, adapters, rank, order, none, ragged, dtype):
    return {"name": name, "op": "low_rank_add", "tokens": tokens, "ch": ch, "m": m, "adapters": adapters, "rank": rank,
            "order": order, "none": none, "ragged": ragged, "dtype": dtype}


def _mass(name, batch, new, past, ragged, heads, kv_heads, dim, dtype, page, order, window=0, causal=True, mix=1):
    return {"name": name, "op": "attention_mass", "batch": batch, "new": new, "past": past, "ragged": ragged,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page, "order": order,
            "window": window, "causal": causal, "mix": mix}


def _evict(name, batch, length, ragged, over, kv_heads, dim, dtype, page, order, first, recent, positions, mix=1):
    return {"name": name, "op": "evict", "batch": batch, "length": length, "ragged": ragged, "over": over,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page, "order": order, "first": first,
            "recent": recent, "positions": positions, "mix": mix}


def listed():
    return [
        # one generated token of one request
        _adapt("adapt_one_token_bf16", 1, 4096, 6144, 8, 16, "mixed", 0.0, False, "bf16"),
        # one generated token of each of 64 requests, nearly as many adapters, some requests with none
        _adapt("adapt_batch_bf16", 64, 4096, 6144, 48, 32, "mixed", 0.15, False, "bf16"),
        # prompts of six requests, one after the other
        _adapt("adapt_prompts_bf16", 8192, 4096, 4096, 6, 64, "runs", 0.0, False, "bf16"),
        # an odd count of tokens in any order, ranks that differ, sizes that no tile divides
        _adapt("adapt_odd_f32", 517, 1000, 1288, 5, 24, "mixed", 0.2, True, "f32"),
        # the first generated tokens of a short chat
        _mass("mass_short_bf16", 1, 1, 76, False, 32, 8, 128, "bf16", 16, "heads"),
        # a serving batch: one token each, contexts of very different lengths, one place unused
        _mass("mass_batch_bf16", 64, 1, 8191, True, 32, 8, 128, "bf16", 16, "heads"),
        # two whole prompts
        _mass("mass_prompts_bf16", 2, 8192, 0, False, 32, 8, 128, "bf16", 64, "heads"),
        # fp32 with a sliding window, odd lengths, pages of 24 rows, heads inside rows
        _mass("mass_window_f32", 3, 257, 1000, False, 12, 4, 64, "f32", 24, "rows", window=512),
        # a generated token of each of 64 requests whose caches are full: one row out for each
        _evict("evict_step_bf16", 64, 4097, False, 1 / 4097, 8, 128, "bf16", 16, "heads", 4, 256, True),
        # prompts just read, cut down to an eighth
        _evict("evict_prompts_bf16", 8, 8192, True, 7 / 8, 8, 128, "bf16", 64, "heads", 16, 512, False),
        # one very long context, halved
        _evict("evict_long_bf16", 1, 131072, False, 1 / 2, 8, 128, "bf16", 64, "heads", 4, 1024, True),
        # fp32, odd lengths, pages of 24 rows, heads inside rows, some sequences within their budget
        _evict("evict_ragged_f32", 13, 1571, True, 0.3, 5, 80, "f32", 24, "rows", 0, 33, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    return {k: v for k, v in _drawn(rng).items() if k != "name"}


def _drawn(rng):
    op = rng.choice(["low_rank_add", "attention_mass", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "low_rank_add":
        while True:
            c = _adapt("", _log(rng, 1, 16384), 8 * _log(rng, 4, 1024), 8 * _log(rng, 4, 1024), _log(rng, 1, 64),
                       8 * rng.randint(1, 16), rng.choice(["runs", "mixed"]), rng.choice([0.0, 0.0, 0.3]),
                       rng.random() < 0.3, dtype)
            # the plain form multiplies every token by every adapter
            if (2.0 * c["tokens"] * c["adapters"] * c["rank"] * (c["ch"] + c["m"]) <= MAX_ADAPT and
                    c["tokens"] * (c["ch"] + 2.0 * c["m"]) <= MAX_ROWS):
                return c
    dim = rng.choice([64, 96, 128, 128, 128, 192, 256, 8 * rng.randint(4, 32)])
    kv_heads = rng.choice([1, 2, 4, 8, 8, rng.randint(3, 12)])
    page = rng.choice([16, 16, 32, 64, 128, rng.randint(5, 200)])
    order = rng.choice(["heads", "rows"])
    if op == "evict":
        while True:
            batch, length = _log(rng, 1, 128), _log(rng, 2, 131072)
            # one row out, as in each step of a full cache, or a part of them
            over = rng.choice([1.0 / length, rng.uniform(0.05, 0.95)])
            if batch * kv_heads * length * dim <= MAX_CACHE:
                return _evict("", batch, length, rng.random() < 0.6, over, kv_heads, dim, dtype, page, order,
                              rng.choice([0, 4, 16]), rng.choice([0, 64, 512]), rng.random() < 0.5,
                              rng.randint(0, 1 << 20))
    heads = kv_heads * rng.choice([1, 2, 4, 4, 8, rng.randint(1, 8)])
    while True:
        new = 1 if rng.random() < 0.5 else _log(rng, 2, 8192)
        past = _log(rng, 1, 131072) - 1
        batch = _log(rng, 1, 128)
        window = rng.choice([0, 0, 0, _log(rng, 16, 8192)])
        c = _mass("", batch, new, past, rng.random() < 0.6, heads, kv_heads, dim, dtype, page, order, window,
                  window > 0 or rng.random() < 0.9, rng.randint(0, 1 << 20))
        # the plain form works on sequences padded to the longest
        length, top = past + new, MAX_SCORES if dtype == "bf16" else MAX_SCORES / 8
        if batch * heads * new * length > top or batch * kv_heads * length * dim > MAX_CACHE:
            continue
        if work(c)["flops"] <= (MAX_FLOPS if dtype == "bf16" else MAX_FLOPS / 8):
            return c


def _lengths(c):
    """attention_mass: new tokens and cached tokens (the new ones among them) of each sequence.  evict: cached
    tokens, and those that are to stay.  Ragged: the first sequence is the longest, and of four or more the last
    is an unused place; every fifth that is to be cut is within its budget instead."""
    rng = random.Random(c["mix"])
    one, two = [], []
    for b in range(c["batch"]):
        unused = c["ragged"] and b == c["batch"] - 1 and b >= 3
        if c["op"] == "evict":
            n = _log(rng, 1, c["length"]) if c["ragged"] and b else c["length"]
            n = 0 if unused else n
            k = n - max(1, int(round(n * c["over"])))
            one.append(n)
            two.append(n + 7 if c["ragged"] and b % 5 == 4 else max(k, 0))
            continue
        n, p = c["new"], c["past"]
        if c["ragged"] and b:
            n, p = _log(rng, 1, n), _log(rng, 1, p + 1) - 1
        if unused:
            n, p = (1 if c["new"] == 1 else 0), 0
        one.append(n)
        two.append(0 if unused else n + p)
    return one, two


def _cache(g, c, pages):
    """Pages of keys or values as [page][row][head][dim]; in memory a page holds its heads one after
    the other ("heads") or its rows ("rows")."""
    dt = DTYPES[c["dtype"]]
    if c["order"] == "heads":
        shape = (pages, c["kv_heads"], c["page"], c["dim"])
        return torch.randn(shape, generator=g, device="cuda").to(dt).transpose(1, 2)
    return torch.randn((pages, c["page"], c["kv_heads"], c["dim"]), generator=g, device="cuda").to(dt)


def _pages(g, c, length):
    """Every sequence's pages in any order, [batch][entries]; page 0 belongs to nobody: unused entries name it."""
    count = [-(-n // c["page"]) for n in length]
    order = torch.randperm(sum(count), generator=g, device="cuda") + 1
    pages = torch.zeros(c["batch"], max(1, max(count)), dtype=torch.int32)
    place = torch.zeros(pages.shape, dtype=torch.bool)
    for b, n in enumerate(count):
        place[b, :n] = True
    pages = pages.cuda()
    pages[place.cuda()] = order.int()
    return pages, sum(count) + 1


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    s = {"case": c}
    if c["op"] == "low_rank_add":
        t, n, r = c["tokens"], c["adapters"], c["rank"]
        s["x"], s["y"] = normal(t, c["ch"]), normal(t, c["m"])
        s["a"] = normal(n, r, c["ch"], scale=c["ch"] ** -0.5)
        s["b"] = normal(n, c["m"], r, scale=r ** -0.5)
        s["scales"] = 0.25 + torch.rand(n, generator=g, device="cuda")
        s["ranks"] = None
        if c["ragged"]:
            s["ranks"] = torch.randint(1, r + 1, (n,), generator=g, device="cuda").int()
        if c["order"] == "runs":
            ids = (torch.arange(t, device="cuda") * n // t + torch.randint(0, n, (1,), generator=g, device="cuda")) % n
        else:
            ids = torch.randint(0, n, (t,), generator=g, device="cuda")
        off = torch.rand(t, generator=g, device="cuda") < c["none"]
        s["ids"] = torch.where(off, -1, ids).int()
        return s
    if c["op"] == "attention_mass":
        new, length = _lengths(c)
        s["pages"], count = _pages(g, c, length)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        s["q"] = normal(starts[-1], c["heads"], c["dim"])
        s["k_cache"] = _cache(g, c, count)
        s["kv_lens"] = torch.tensor(length, dtype=torch.int32, device="cuda")
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["max_q"], s["max_kv"] = max(new), max(length)
        # what earlier steps left, about as much as these tokens bring, and the log-sums that their attention gave
        s["mass"] = torch.rand((c["batch"], s["pages"].shape[1] * c["page"]), generator=g, device="cuda")
        s["mass"] *= c["heads"] * c["new"] / s["max_kv"]
        s["lse"] = torch.logsumexp(_scores(s), -1)[_rows(s)].reshape(starts[-1], c["heads"]).contiguous()
        return s
    length, keep = _lengths(c)
    s["pages"], count = _pages(g, c, length)
    s["k_cache"], s["v_cache"] = _cache(g, c, count), _cache(g, c, count)
    s["kv_lens"] = torch.tensor(length, dtype=torch.int32, device="cuda")
    s["keep"] = torch.tensor(keep, dtype=torch.int32, device="cuda")
    s["max_kv"] = max(length)
    places = s["pages"].shape[1] * c["page"]
    # a few keys get most of the weight
    s["mass"] = torch.randn((c["batch"], places), generator=g, device="cuda").mul_(2.0).exp_()
    s["positions"] = None
    if c["positions"]:   # rows that earlier calls moved lie anywhere but for the latest
        spread = torch.rand((c["batch"], places), generator=g, device="cuda") * 64
        p = torch.arange(places, device="cuda") + spread
        s["positions"] = p.argsort(1).argsort(1).int()
    s["since"] = (s["kv_lens"] - c["recent"]).int()
    return s


# ---- the plain forms --------------------------------------------------------------------------

def _plain_adapt(s):
    c = s["case"]
    t, n, r = c["tokens"], c["adapters"], c["rank"]
    a, b = s["a"].float().view(n * r, c["ch"]), s["b"].float().transpose(1, 2).reshape(n * r, c["m"])
    h = torch.matmul(s["x"].float(), a.t()).view(t, n, r)
    mine = (s["ids"][:, None] == torch.arange(n, device=h.device))[:, :, None]
    if s["ranks"] is not None:
        mine = mine & (torch.arange(r, device=h.device) < s["ranks"][:, None])
    h = torch.where(mine, h * s["scales"][:, None], 0.0).view(t, n * r)
    return {"out": (s["y"].float() + torch.matmul(h, b)).to(s["y"].dtype)}


def _scores(s):
    """Scores of every new token and cached key, [batch][kv_heads][group][new][places] in 32 bits, -infinity
    where a row does not see a key."""
    c = s["case"]
    heads, kv, d = c["heads"], c["kv_heads"], c["dim"]
    q, lens, starts = s["q"], s["kv_lens"].long(), s["q_starts"].long()
    batch, tokens, mq, group = lens.shape[0], q.shape[0], s["max_q"], heads // kv
    new = starts[1:] - starts[:-1]
    pages = s["pages"].long()
    length = pages.shape[1] * c["page"]
    K = s["k_cache"][pages].float().reshape(batch, length, kv, d).transpose(1, 2)
    i = torch.arange(mq, device=q.device)
    Q = q[(starts[:-1, None] + i).clamp(max=tokens - 1)].float()            # [batch][mq][heads][d]
    Q = Q.view(batch, mq, kv, group, d).permute(0, 2, 3, 1, 4).reshape(batch, kv, group * mq, d)
    S = torch.matmul(Q, K.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d))
    at = (lens - new)[:, None] + i                                            # positions [batch][mq]
    j = torch.arange(length, device=q.device)
    hide = (j >= lens[:, None])[:, None] | (i >= new[:, None])[:, :, None]
    if c["causal"]:
        hide = hide | (j > at[:, :, None])
    if c["window"]:
        hide = hide | (j <= at[:, :, None] - c["window"])
    return S.view(batch, kv, group, mq, length).masked_fill_(hide[:, None, None], -math.inf)


def _rows(s):
    """The indices [batch, kv_heads, group, new] of every token's heads, [tokens][kv_heads][group]."""
    c, starts = s["case"], s["q_starts"].long()
    kv, group = c["kv_heads"], c["heads"] // c["kv_heads"]
    t = torch.arange(s["q"].shape[0], device=starts.device)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    h, x = torch.arange(kv, device=t.device), torch.arange(group, device=t.device)
    return b[:, None, None], h[:, None], x, (t - starts[b])[:, None, None]


def _plain_mass(s):
    c = s["case"]
    S = _scores(s)
    lse = torch.zeros(S.shape[:-1], device=S.device)
    lse[_rows(s)] = s["lse"].view(-1, c["kv_heads"], c["heads"] // c["kv_heads"])
    lse = torch.where(lse == -math.inf, 0.0, lse)                             # a row that sees nothing
    s["mass"] += S.sub_(lse.unsqueeze(-1)).exp_().sum((1, 2, 3))
    return {"mass": s["mass"]}


def _plain_evict(s):
    c = s["case"]
    pages = s["pages"].long()
    batch, places = pages.shape[0], pages.shape[1] * c["page"]
    j = torch.arange(places, device=pages.device).expand(batch, places)
    n = s["kv_lens"].long()[:, None]
    k = torch.minimum(s["keep"].long()[:, None], n)
    positions = s["positions"] if s["positions"] is not None else j.int()
    kept_for = (positions < c["first"]) | (positions >= s["since"][:, None])
    # first by whether a row is kept for its position, then by weight, then by place; rows that are not there last
    order = s["mass"].argsort(dim=1, descending=True, stable=True)
    order = order.gather(1, kept_for.gather(1, order).long().argsort(dim=1, descending=True, stable=True))
    order = order.gather(1, (j < n).gather(1, order).long().argsort(dim=1, descending=True, stable=True))
    rank = torch.empty_like(order).scatter_(1, order, j)
    stays = rank < k
    free, moves = ~stays & (j < k), stays & (j >= k)
    half = places // 2 + 1
    to = free.long().argsort(dim=1, descending=True, stable=True)[:, :half]
    at = moves.long().argsort(dim=1, descending=True, stable=True)[:, :half]
    some = j[:, :half] < moves.sum(1, keepdim=True)

    def row(x):   # page 0's first row, which is nobody's, moves onto itself
        return torch.where(some, pages.gather(1, x // c["page"]), 0), torch.where(some, x % c["page"], 0)

    for cache in (s["k_cache"], s["v_cache"]):
        cache[row(to)] = cache[row(at)]
    source = j.clone().scatter_(1, to, torch.where(some, at, to))
    there = j < k
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": k[:, 0].int(),
            "mass": torch.where(there, s["mass"].gather(1, source), 0.0),
            "positions": torch.where(there, positions.gather(1, source), -1)}


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "low_rank_add":
            return _plain_adapt(s)
        return _plain_mass(s) if c["op"] == "attention_mass" else _plain_evict(s)
    from paper_2003_12203_amd import adapters, paged
    if c["op"] == "low_rank_add":
        return {"out": adapters.low_rank_add(s["y"], s["x"], s["a"], s["b"], s["ids"], s["scales"], s["ranks"])}
    if c["op"] == "attention_mass":
        paged.attention_mass(s["mass"], s["q"], s["k_cache"], s["pages"], s["kv_lens"], s["lse"],
                             None if c["new"] == 1 else s["q_starts"], s["max_q"], s["max_kv"], causal=c["causal"],
                             window=c["window"])
        return {"mass": s["mass"]}
    lens, mass, positions = paged.evict(s["k_cache"], s["v_cache"], s["pages"], s["kv_lens"], s["keep"], s["mass"],
                                        s["positions"], c["first"], s["since"], s["max_kv"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": lens, "mass": mass, "positions": positions}


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "low_rank_add":
        used = c["adapters"] * (1.0 - (1.0 - (1.0 - c["none"]) / c["adapters"]) ** c["tokens"])   # drawn at random
        if c["order"] == "runs":
            used = min(c["adapters"], c["tokens"])
        mine, rank = c["tokens"] * (1.0 - c["none"]), c["rank"] * (0.5 if c["ragged"] else 1.0)
        return {"bytes": es * (mine * c["ch"] + 2.0 * c["tokens"] * c["m"] + used * rank * (c["ch"] + c["m"]))
                + 4.0 * c["tokens"], "flops": 2.0 * mine * rank * (c["ch"] + c["m"])}
    one, two = _lengths(c)
    if c["op"] == "evict":
        moved = sum((n - k) * k / n for n, k in zip(one, two) if k < n)
        return {"bytes": moved * 4.0 * es * c["kv_heads"] * c["dim"]
                + sum(one) * (16.0 if c["positions"] else 12.0), "flops": 1.0 * sum(one)}
    d = c["dim"]
    pairs = rows = 0
    for n, m in zip(one, two):
        if not n or not m:
            continue
        w = c["window"] or m
        if not c["causal"]:
            pairs += n * m
            rows += m
            continue
        past = m - n
        # position p sees min(p + 1, w) keys
        full = max(0, min(n, w - past))          # rows that see every key before them
        pairs += full * past + full * (full + 1) // 2 + (n - full) * w
        rows += min(m, w + n - 1)
    t = sum(one)
    return {"bytes": es * (1.0 * t * c["heads"] * d + rows * c["kv_heads"] * d) + 4.0 * t * c["heads"] + 8.0 * rows
            + 4.0 * rows / c["page"], "flops": 2.0 * pairs * c["heads"] * d}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "low_rank_add":
        out, ids = s["y"].double(), s["ids"].tolist()
        for a in sorted(set(ids) - {-1}):
            mine = s["ids"] == a
            r = c["rank"] if s["ranks"] is None else int(s["ranks"][a])
            low = s["x"][mine].double() @ s["a"][a, :r].double().t().contiguous()
            out[mine] += float(s["scales"][a]) * (low @ s["b"][a, :, :r].double().t().contiguous())
        return {"out": out}
    one, two = _lengths(c)
    page = c["page"]
    if c["op"] == "attention_mass":
        mass, t = s["mass"].double(), 0
        d, group = c["dim"], c["heads"] // c["kv_heads"]
        for b, (n, m) in enumerate(zip(one, two)):
            mine = s["pages"][b, :-(-m // page)].long()
            for h in range(c["kv_heads"] if n and m else 0):
                K = s["k_cache"][mine, :, h].reshape(-1, d)[:m].double().t().contiguous()
                step = max(1, int(4e8 // m))                       # rows at a time
                for r in range(h * group, (h + 1) * group):
                    for a in range(0, n, step):
                        e = min(n, a + step)
                        S = (s["q"][t + a:t + e, r].double() @ K) / math.sqrt(d)
                        p = torch.arange(m - n + a, m - n + e, device=S.device)[:, None]
                        j = torch.arange(m, device=S.device)[None]
                        seen = (j <= p) if c["causal"] else torch.ones_like(j <= p)
                        if c["window"]:
                            seen = seen & (j > p - c["window"])
                        w = torch.exp(S - s["lse"][t + a:t + e, r, None].double())
                        mass[b, :m] += torch.where(seen, w, 0.0).sum(0)
            t += n
        return {"mass": mass}
    out = {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double(),
           "lens": torch.tensor([min(n, k) for n, k in zip(one, two)], dtype=torch.int32, device="cuda"),
           "mass": torch.zeros(s["mass"].shape, dtype=torch.float64, device="cuda"),
           "positions": torch.full(s["mass"].shape, -1, dtype=torch.int32, device="cuda")}
    for b, (n, k) in enumerate(zip(one, two)):
        k = min(n, k)
        w = s["mass"][b, :n].tolist()
        p = s["positions"][b, :n].tolist() if s["positions"] is not None else list(range(n))
        best = sorted(range(n), key=lambda j: (not (p[j] < c["first"] or p[j] >= n - c["recent"]), -w[j], j))[:k]
        holes, late = sorted(set(range(k)) - set(best)), sorted(j for j in best if j >= k)
        now = list(range(k))
        for to, at in zip(holes, late):
            now[to] = at
        if holes:
            lists = s["pages"][b].long()
            to, at = torch.tensor(holes, device="cuda"), torch.tensor(late, device="cuda")
            for name in ("k_cache", "v_cache"):
                out[name][lists[to // page], to % page] = out[name][lists[at // page], at % page]
        if k:
            out["mass"][b, :k] = torch.tensor([w[j] for j in now], dtype=torch.float64, device="cuda")
            out["positions"][b, :k] = torch.tensor([p[j] for j in now], dtype=torch.int32, device="cuda")
    return out
