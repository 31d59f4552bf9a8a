"""Queries, keys and values that are not finite in pc_attn_paged, over caches of one
range and of many: what a row sees reaches its result as NaN, statistics and weights
too, and nothing else; only a row that sees nothing has zeros."""
import numpy as np
import pytest
import torch

from test_attn_gpu import BF16, F16, FP8, Case
from paper_2609_28870_amd import pc

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, FP8)], ids=["bf16", "f16", "fp8"])


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def visible(c, s, causal=True, window=0):
    """[new row, slot] of sequence s: what each row sees."""
    n, m = int(c.kv[s]), int(c.new[s])
    x, j = n - m + np.arange(m)[:, None], np.arange(n)[None]
    see = np.ones((m, n), bool)
    if causal:
        see &= j <= x
    if window:
        see &= j > x - window
    return see


def compare(got, want, tol, spoilt_rows, spoilt_slots):
    """Results against those of finite inputs: NaN where a spoilt row or slot says so, the
    others within their bounds."""
    for name, x, y, t, bad in zip(("out", "lse", "weight"), got, want, tol, (spoilt_rows, spoilt_rows, spoilt_slots)):
        x = x.detach().cpu().double().numpy()
        assert np.isnan(x[bad]).all(), name
        ok = ~bad & np.ones(x.shape[:bad.ndim], bool)
        none = np.isinf(y[ok])
        assert np.array_equal(x[ok][none], y[ok][none]), name
        over = np.abs(x[ok][~none] - y[ok][~none]) - t[ok][~none]
        assert over.size == 0 or over.max() <= 0, (name, float(over.max()))


@pytest.mark.parametrize("new", [1, 4, 64])
@pytest.mark.parametrize("window", [0, 1500])
@TYPES
def test_a_row_of_a_broken_query(new, window, dtype, cache):
    """Sequences of one range of keys and of twenty: out, lse and the weights of what the row sees."""
    c = Case([5000, 90], [new, new], heads=8, kvh=2, dtype=dtype, cache=cache, seed=new, weights=True)
    want, tol = c.want(window=window)
    rows, slots = np.zeros((2 * new, 8), bool), np.zeros(c.weight.shape, bool)
    for s, i, e in ((0, new // 2, 5), (1, new - 1, 2)):
        c.q[s * new + i, e, 3] = float("nan")
        rows[s * new + i, e] = True
        slots[s, e // 4, :c.kv[s]] = visible(c, s, window=window)[i]
    got = c.run(window=window)
    torch.cuda.synchronize()
    assert pc.workspace_status(got[3]) == 0
    compare(got, want, tol, rows, slots)


@pytest.mark.parametrize("kv,new,window", [(5000, 1, 0), (5000, 4, 0), (5000, 64, 0), (5000, 64, 3500), (2600, 1500, 0),
                                           (2600, 1500, 600)])
@TYPES
def test_a_range_of_broken_keys(kv, new, window, dtype, cache):
    """Every key of some whole ranges is NaN: rows that see any of them are, and no other."""
    c = Case([kv], [new], heads=4, kvh=2, dtype=dtype, cache=cache, seed=kv + new, weights=True)
    want, tol = c.want(window=window)
    lo, hi = 1024, 2048 if kv == 5000 else 1600
    pages = torch.from_numpy(c.table[0, lo // 16:hi // 16]).cuda()
    if cache == FP8:
        c.kc.view(torch.uint8)[pages, 1] = 0x7F
    else:
        c.kc[pages, 1] = float("nan")
    see = visible(c, 0, window=window)
    hit = see[:, lo:hi].any(1)
    rows, slots = np.zeros((new, 4), bool), np.zeros(c.weight.shape, bool)
    rows[:, 2:] = hit[:, None]
    slots[0, 1, :kv] = see[hit].any(0)
    assert hit.any() or window
    compare(c.run(window=window), want, tol, rows, slots)


@pytest.mark.parametrize("new,others", [(4, 99), (64, 39)])
@TYPES
def test_one_of_few_parts_of_broken_keys(new, others, dtype, cache):
    """One of three ranges, in a batch so large that a join takes all of a row's parts at once."""
    c = Case([700] + [9] * others, [new] + [min(new, 9)] * others, heads=32, kvh=4, dtype=dtype, cache=cache, seed=new,
             weights=True)
    want, tol = c.want()
    pages = torch.from_numpy(c.table[0, 16:32]).cuda()
    if cache == FP8:
        c.kc.view(torch.uint8)[pages, 1] = 0x7F
    else:
        c.kc[pages, 1] = float("nan")
    rows, slots = np.zeros((c.q.shape[0], 32), bool), np.zeros(c.weight.shape, bool)
    rows[:new, 8:16] = True
    slots[0, 1, :700] = True
    compare(c.run(), want, tol, rows, slots)


@pytest.mark.parametrize("new", [1, 64])
def test_a_broken_range_among_rows_that_see_nothing(new):
    """Rows before the first slot see nothing, and stay zeros beside broken ones."""
    c = Case([max(3, new - 20), 5000], [new + 4, new], heads=4, kvh=1, seed=new, weights=True)
    c.q[-1] = float("nan")
    out, lse, weight, ws = c.run()
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == (2 if new + 4 > int(c.kv[0]) else 0)
    none = max(0, new + 4 - int(c.kv[0]))
    assert bool((out[:none] == 0).all()) and bool((lse[:none] == -float("inf")).all())
    assert bool(torch.isfinite(out[none:-1]).all()) and bool(torch.isfinite(lse[none:-1]).all())
    assert bool(torch.isnan(out[-1]).all()) and bool(torch.isnan(lse[-1]).all())
    assert bool(torch.isfinite(weight[0]).all()) and bool(torch.isnan(weight[1, 0, :5000]).all())
    assert bool((weight[1, :, 5000:] == 0).all())


@pytest.mark.parametrize("new", [1, 64])
@pytest.mark.parametrize("kv", [90, 5000])
def test_scores_of_minus_infinity_weigh_nothing(new, kv):
    """A row whose every score is -infinity is one that sees nothing: exp(-infinity) = 0, however its keys are cut."""
    c = Case([kv], [new], heads=4, kvh=2, seed=kv, weights=True)
    c.q.abs_()
    c.kc[:, 0, :, 5] = -float("inf")
    want, tol = c.want()
    out, lse, weight, _ = c.run()
    torch.cuda.synchronize()
    assert bool((out[:, :2] == 0).all()) and bool((lse[:, :2] == -float("inf")).all())
    assert torch.equal(weight[0, 0, :kv], c.weight[0, 0, :kv])
    for x, y, t in ((out[:, 2:], want[0][:, 2:], tol[0][:, 2:]), (lse[:, 2:], want[1][:, 2:], tol[1][:, 2:]),
                    (weight[:, 1], want[2][:, 1], tol[2][:, 1])):
        assert np.all(np.abs(x.cpu().double().numpy() - y) <= t)


@pytest.mark.parametrize("new", [1, 64])
@pytest.mark.parametrize("kv", [90, 5000])
@TYPES
@pytest.mark.parametrize("broken", [float("nan"), float("inf")])
def test_a_factor_of_zero_keeps_a_broken_query_broken(new, kv, dtype, cache, broken):
    """0 * NaN and 0 * infinity are NaN: by a scale of zero, or an 8-bit cache's scale of zero."""
    c = Case([kv], [new], heads=4, kvh=2, dtype=dtype, cache=cache, seed=kv, weights=True)
    scale = 0.0
    if cache == FP8:
        c.ks[0], scale = 0.0, 0.2
    want, tol = c.want(scale=scale)
    rows, slots = np.zeros((new, 4), bool), np.zeros(c.weight.shape, bool)
    c.q[new // 2, 1, 3] = broken
    rows[new // 2, 1] = True
    slots[0, 0, :kv] = visible(c, 0)[new // 2]
    compare(c.run(scale=scale), want, tol, rows, slots)
