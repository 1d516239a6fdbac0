"""Every instance that attention over the paged cache is compiled for, against its definition in float64: a kernel for up
to 16 rows of a key head or for more, columns of 64, 128 and 256, whole units or even runs, one page to a
wave's loads or several.  Each case says which schedule it takes, and the library's plan is asked."""
import numpy as np
import pytest

from oracle import serving as sv
from test_gpu_paged import attend, batch, check, f64, near
from test_gpu_paged_limits import is_split

pytestmark = pytest.mark.gpu

DIMS = [64, 40, 128, 104, 256, 192, 136]
WIDE = {False: ([70, 20, 33], [90, 20, 33]), True: ([40, 1], [3000, 900])}
FEW = {False: ([1, 3], [40, 19]), True: ([2, 1], [2500, 70])}


def run(dtype, dim, page, split, new, length, heads, kv, **kw):
    rng = np.random.default_rng([dim, page, sum(length)])
    args = batch(rng, new, length, heads, kv, dim, dtype, page, fill=float("nan"))
    assert is_split(args[0], args[1], args[3], new, length, **kw) == split
    check(*args, dtype, max_q=max(new), max_kv=max(length), **kw)


@pytest.mark.parametrize("page", [16, 8, 7])     # 7, and 8 in bf16 up to 128: a wave's loads lie in several pages
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_than_16_rows(dtype, dim, split, page):
    run(dtype, dim, page, split, *WIDE[split], heads=2, kv=1)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_up_to_16_rows(dtype, dim, split):
    run(dtype, dim, 16, split, *FEW[split], heads=4, kv=1)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_windows(dtype, dim):
    """A window over both schedules of workgroups, its tiles masked at both ends."""
    run(dtype, dim, 7, False, [70, 20], [300, 20], heads=2, kv=1, window=45)
    run(dtype, dim, 16, True, [40], [3000], heads=2, kv=1, window=1500)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wide_groups(dtype):
    """One new token each of more than 16 query heads to a key head: rows of the kernel for many."""
    run(dtype, 64, 16, False, [1, 1], [200, 31], heads=24, kv=1)
    run(dtype, 128, 16, True, [1, 1], [3000, 70], heads=20, kv=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(128, 16), (120, 7), (256, 16), (200, 7)])
@pytest.mark.parametrize("new,length,window", [(70, 100, 0), (40, 3000, 0), (70, 300, 45), (1, 50, 0), (2, 2500, 2000)])
def test_infinities_and_nan_reach_the_rows_that_see_them(dtype, dim, page, new, length, window):
    """Among the last keys, and among the first, which a window may have left."""
    rng = np.random.default_rng([dim, length])
    q, kc, vc, lists, lens, starts = batch(rng, [new], [length], 2, 1, dim, dtype, page)
    for cache, j, at, x in ((vc, length - 2, 3, float("inf")), (vc, length - 2, 5, float("-inf")),
                            (vc, length - 1, 5, float("inf")), (vc, length - 3, dim - 1, float("nan")),
                            (vc, 1, dim - 2, float("inf")), (vc, length - new // 2 - 1, 9, float("-inf")),
                            (kc, length - 1, 1, float("nan") if new > 1 else 0.0)):
        cache[lists[0, j // page], j % page, 0, at] = x
    got = attend(q, kc, vc, lists, lens, starts, window=window, max_q=new, max_kv=length)
    want = sv.attention(f64(q), f64(kc), f64(vc), lists, lens, starts, None, True, window, dtype)
    near(got[0], want[0], np.nan_to_num(want[2], nan=0.0, posinf=0.0), "out")
    near(got[1], want[1], np.nan_to_num(want[3], nan=0.0, posinf=0.0), "lse")
    assert np.isfinite(want[0]).any()
