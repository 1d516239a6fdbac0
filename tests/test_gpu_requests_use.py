"""Adapters, attention mass and eviction together in a served layer (examples/served_requests.py)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("served_requests", os.path.join(ROOT, "examples", "served_requests.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_a_budget(example, dtype):
    """The layer's outputs, and every row's weights add up to 1 for each head."""
    res = example.serve(dtype, new=5)
    # Rounding as in the layer alone: in bf16, queries and keys of unit size are off by 2^-8 each, a score (a sum of 64 such
    # products, scaled) by about 2^-7, outputs by a few percent, their largest of some 10^5 by four times that; in fp32, 2^-16
    # of these.  An adapter that is another's, or missing, is off by more than one.
    assert res["worst"] < (0.5 if dtype == "bf16" else 1e-3) and res["gone"] == 0
    mass, heads = res["state"].mass.double(), res["layer"].heads
    for b, n in enumerate(res["total"]):
        # fp32: sums of up to 2000 terms (2^-24 each), scores of up to 10 as sums of 64 products in two orders (2^-18 each
        # at most), log-sums of up to 16 (2^-21)
        assert abs(float(mass[b].sum()) / (heads * n) - 1.0) < 1e-4
        assert mass[b, n:].eq(0).all() and mass[b, :n].gt(0).all()
    positions = res["state"].positions
    assert all(positions[b, :n].tolist() == list(range(n)) for b, n in enumerate(res["total"]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_within_a_budget(example, dtype):
    res = example.serve(dtype, budget=70, new=9)
    state, total = res["state"], res["total"]
    lens = [min(t, 70) for t in total]
    assert state.sequences.lens == lens and res["gone"] == sum(total) - sum(lens)
    held = sum(-(-n // state.sequences.page) for n in lens)
    assert len(state.sequences.free) + held == res["layer"].cache.pages   # no page lost, none twice
    names = state.sequences.free + [int(p) for b, n in enumerate(lens) for p in state.sequences.lists[b, :-(-n // state.sequences.page)]]
    assert sorted(names) == list(range(res["layer"].cache.pages))
    for b, (n, t) in enumerate(zip(lens, total)):
        p = state.positions[b, :n].tolist()
        assert len(set(p)) == n and all(0 <= x < t for x in p)
        assert set(range(4)) <= set(p) and set(range(t - 16, t)) <= set(p)
        assert state.positions[b, n:].eq(-1).all() and state.mass[b, n:].eq(0).all() and state.mass[b, :n].gt(0).all()
    assert all(torch.isfinite(o).all() for o in res["outs"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_until_something_is_taken_out(example, dtype):
    """A budget of all tokens changes no bit; a smaller one none before it is reached, in the step that reads tokens 96 to 143
    of the longest prompt (the others then have 39 and 65)."""
    whole, same, some = (example.serve(dtype, new=5, budget=n) for n in (None, 205, 120))
    assert same["gone"] == 0 and all(torch.equal(a, b) for a, b in zip(whole["outs"], same["outs"]))
    assert some["gone"] == 205 - 120
    assert all(torch.equal(whole["outs"][b][:n], some["outs"][b][:n]) for b, n in enumerate((144, 39, 65)))
