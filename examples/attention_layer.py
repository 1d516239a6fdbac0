"""One attention layer served token by token: protected projections, norms and rotation, a paged cache,
attention.

    python examples/attention_layer.py [--dtype f32] [--new 24]

Three prompts of different lengths are read in chunks and then continued by single tokens.  The two
projections are checksum-protected layers of 1x1 maps with the tokens as the batch; one of each step's
values is disturbed on purpose and corrected.  Between them are the operators of
``paper_2003_12203_amd.paged``.  Every step's output is compared with the layer in float64.
"""
from __future__ import annotations

import argparse
import os
import sys
from typing import List, Sequence

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2003_12203_amd as ft  # noqa: E402
from paper_2003_12203_amd import paged  # noqa: E402


class Sequences:
    """Which pages each sequence holds, and the index arrays of a step."""

    def __init__(self, count: int, pages: int, page: int, entries: int):
        self.page, self.free = page, list(range(pages))
        self.lens = [0] * count
        self.lists = torch.zeros(count, entries, dtype=torch.int32)

    def step(self, new: Sequence[int], device="cuda") -> dict:
        """Room for new[b] more tokens of each sequence, and the arrays that the operators take."""
        seq, positions, starts = [], [], [0]
        for b, n in enumerate(new):
            held, want = -(-self.lens[b] // self.page), -(-(self.lens[b] + n) // self.page)
            for e in range(held, want):
                self.lists[b, e] = self.free.pop()
            seq += [b] * n
            positions += range(self.lens[b], self.lens[b] + n)
            starts.append(starts[-1] + n)
            self.lens[b] += n
        i32 = dict(dtype=torch.int32, device=device)
        return dict(seq=torch.tensor(seq, **i32), positions=torch.tensor(positions, **i32),
                    q_starts=torch.tensor(starts, **i32), kv_lens=torch.tensor(self.lens, **i32),
                    page_list=self.lists.to(device), max_q=max(new), max_kv=max(self.lens))


class AttentionLayer:
    """x [tokens][hidden] -> [tokens][hidden]: a packed projection to queries, keys and values, their norms
    and rotation, attention over the cache, a projection back."""

    def __init__(self, hidden, heads, kv_heads, dim, cache: paged.PagedCache, max_pos, dtype="bf16", seed=0):
        self.hidden, self.heads, self.kv_heads, self.dim, self.dtype = hidden, heads, kv_heads, dim, dtype
        rng = torch.Generator().manual_seed(seed)
        tdt = ft.DTYPES[dtype][1]

        def weight(m, ch):
            return (torch.randn(m, ch, 1, 1, generator=rng) * ch ** -0.5).to("cuda", tdt)

        self.w_qkv, self.w_out = weight((heads + 2 * kv_heads) * dim, hidden), weight(hidden, heads * dim)
        self.q_weight, self.k_weight = (1.0 + 0.1 * torch.randn(2, dim, generator=rng)).cuda()
        self.table = paged.rope_table(max_pos, dim)
        self.cache = cache
        self.layers = {}

    def _project(self, x, w, faults) -> torch.Tensor:
        """x [tokens][ch] times w [m][ch], checksum-protected: [tokens][m].  The buffers of a size are kept."""
        key = (x.shape[0], w.data_ptr())
        if key not in self.layers:
            # a located value is computed again: the sums of a step's rounded outputs are coarser than one of them
            self.layers[key] = ft.Layer(x.shape[0], w.shape[1], 1, 1, w.shape[0], 1, 1, dtype=self.dtype,
                                        policy=ft.make_policy(repair="recompute"))
            self.layers[key].encode_weights(w)
        layer = self.layers[key]
        out = layer.empty_output()
        layer.protected_fused(x.reshape(layer.shape_d), w, out, faults)
        self.reports.append(layer)
        return out.view(x.shape[0], -1)

    def __call__(self, x, step, faults=((), ())) -> torch.Tensor:
        """One step; faults (testing) are planted in the two projections."""
        self.reports: List[ft.Layer] = []
        h, kv = self.heads, self.kv_heads
        qkv = self._project(x, self.w_qkv, faults[0]).view(-1, h + 2 * kv, self.dim)
        # (places: where a cache whose rows are no longer in the order of their positions takes the new ones)
        slots = self.cache.slots(step["page_list"], step["seq"], step.get("places", step["positions"]))
        q, _ = paged.qk_norm_rope(qkv[:, :h], None, step["positions"], self.table, self.q_weight)
        paged.kv_append(qkv[:, h:h + kv], qkv[:, h + kv:], self.cache.k, self.cache.v, slots, step["positions"],
                        self.table, self.k_weight)
        out = paged.paged_attention(q, self.cache.k, self.cache.v, step["page_list"], step["kv_lens"],
                                    step["q_starts"], step["max_q"], step["max_kv"], lse=step.get("lse"))
        self.qkv, self.q, self.attended = qkv, q, out
        y = self._project(out.view(-1, h * self.dim), self.w_out, faults[1])
        for layer in self.reports:   # the host's one look at a step
            if layer.read_report().status not in (ft.STATUS_CLEAN, ft.STATUS_CORRECTED):
                raise ft.FtcnnError("a projection could not be corrected: the step has to be run again")
        return y

    def plain(self, x: Sequence[torch.Tensor]) -> List[torch.Tensor]:
        """Whole sequences x[b] [tokens][hidden] through the layer in float64 on the CPU, without a cache."""
        def f64(t):
            return t.detach().cpu().double()

        def norm_rope(t, w):
            t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * f64(w)
            c, s = f64(self.table[:t.shape[0], :, 0])[:, None], f64(self.table[:t.shape[0], :, 1])[:, None]
            a, b = t.chunk(2, -1)
            return torch.cat((a * c - b * s, b * c + a * s), -1)

        res = []
        for one in x:
            n, h, kv = one.shape[0], self.heads, self.kv_heads
            qkv = (f64(one) @ f64(self.w_qkv)[:, :, 0, 0].T).view(n, h + 2 * kv, self.dim)
            q, k, v = norm_rope(qkv[:, :h], self.q_weight), norm_rope(qkv[:, h:h + kv], self.k_weight), qkv[:, h + kv:]
            k, v = (t.repeat_interleave(h // kv, 1).transpose(0, 1) for t in (k, v))
            scores = q.transpose(0, 1) @ k.transpose(1, 2) * self.dim ** -0.5
            later = torch.ones(n, n, dtype=torch.bool).triu(1)
            out = torch.softmax(scores.masked_fill(later, -torch.inf), -1) @ v
            res.append(out.transpose(0, 1).reshape(n, -1) @ f64(self.w_out)[:, :, 0, 0].T)
        return res


def serve(dtype="bf16", prompts=(200, 37, 64), chunk=96, new=24, hidden=512, heads=8, kv_heads=2, dim=64, page=16,
          verbose=False):
    """Reads the prompts in chunks of at most `chunk` tokens, then `new` single tokens of each.  Returns the
    largest deviation from the layer in float64, relative to its outputs' root mean square, and the number
    of values corrected."""
    total = [p + new for p in prompts]
    entries = -(-max(total) // page)
    pages = sum(-(-t // page) for t in total)
    cache = paged.PagedCache(pages, page, kv_heads, dim, dtype)
    layer = AttentionLayer(hidden, heads, kv_heads, dim, cache, max(total), dtype)
    rng = torch.Generator().manual_seed(1)
    xs = [torch.randn(t, hidden, generator=rng).to("cuda", ft.DTYPES[dtype][1]) for t in total]
    sequences = Sequences(len(prompts), pages, page, entries)
    outs: List[List[torch.Tensor]] = [[] for _ in prompts]
    corrected = 0
    while sequences.lens != total:
        at = list(sequences.lens)
        now = [min(chunk, p - a) if a < p else min(1, t - a) for a, p, t in zip(at, prompts, total)]
        step = sequences.step(now)
        x = torch.cat([xs[b][a:a + n] for b, (a, n) in enumerate(zip(at, now))])
        fault = dict(n=x.shape[0] // 2, m=17, x=0, y=0, kind="set", value=1e6)
        y = layer(x, step, ((fault,), ()))
        fixes = sum(l.read_report().n_fixes for l in layer.reports)
        corrected += fixes
        if verbose:
            print(f"new {now}  cached {sequences.lens}  corrected {fixes}", flush=True)
        for b, part in enumerate(y.split(now)):
            outs[b].append(part)
    worst = 0.0
    for got, want in zip(outs, layer.plain(xs)):
        got = torch.cat(got).cpu().double()
        worst = max(worst, float((got - want).abs().max() / want.square().mean().sqrt()))
    return worst, corrected


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--dtype", default="bf16", choices=sorted(ft.DTYPES))
    ap.add_argument("--new", type=int, default=24)
    a = ap.parse_args()
    worst, corrected = serve(a.dtype, new=a.new, verbose=True)
    print(f"{a.dtype}: largest deviation from float64 {worst:.2e} of the outputs' root mean square; "
          f"{corrected} values corrected")


if __name__ == "__main__":
    main()
