"""The operators over a paged cache at the ends of their arguments' ranges."""
import numpy as np
import pytest
import torch

from test_attn_gpu import BF16, F16, FP8, Case
from paper_2609_28870_amd import pc

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("scale", [1e-37, 2e-38, -1e-38, 1e-40, -1e-45])
@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_factors_next_to_zero(scale, new, dtype):
    """Weights are then equal to 32 bits: the mean of the values, of one range of keys or of many."""
    Case([100, 41, 3000], [new] * 3, dtype=dtype, weights=True, seed=new).check(scale=scale)


@pytest.mark.parametrize("new", [1, 40])
def test_scales_next_to_zero(new):
    c = Case([100, 41, 3000], [new] * 3, cache=FP8, weights=True, seed=4)
    c.ks[0], c.ks[1] = 1.2e-38, -1e-41
    c.check()


@pytest.mark.parametrize("new", [1, 200])
def test_append_beside_offsets_that_decrease(new):
    """Offsets that decrease in one batch of 64 sequences are reported; the rows of the others, whose
    pages a batch checks together, go where they belong, and a page too many there is reported too."""
    n, page, dim = 150, 16, 16
    off = np.arange(n + 1) * new
    each = (new + page - 1) // page
    table = np.arange(n * each).reshape(n, each)
    rows = torch.randn((n * new, 1, dim), device="cuda").to(BF16)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")   # noqa: E731

    def run(off, table):
        k = torch.zeros((n * each, 1, page, dim), dtype=BF16, device="cuda")
        v = torch.zeros_like(k)
        ws = pc.kv_append(pc.PagedCache(k, v), i32(table), i32([new] * n), i32(off), rows, rows)
        torch.cuda.synchronize()
        assert torch.equal(k, v)
        return pc.workspace_status(ws), k.transpose(1, 2).reshape(n, each * page, 1, dim)
    code, right = run(off, table)
    assert code == 0 and torch.equal(right[:, :new], rows.view(n, new, 1, dim)) and not bool(right[:, new:].any())
    wrong = off.copy()
    wrong[70], wrong[71] = wrong[71], wrong[70]
    code, got = run(wrong, table)
    assert code == 2 and torch.equal(got[:69], right[:69]) and torch.equal(got[72:], right[72:])
    for s in (0, 63, 64, 127, 128, n - 1):
        past = table.copy()
        past[s, -1] = n * each
        assert run(off, past)[0] == 2


@pytest.mark.parametrize("most,long", [(32, 40), (300, 9000)])
def test_append_past_the_bound_writes_no_other_slot(most, long):
    """A length above max_kv is reported: of its new rows those below max_kv go where they
    belong, the others nowhere."""
    page, dim, kv, new = 16, 32, [long, 20], [long - most + 4, 2]
    pages = (long + page - 1) // page + 2
    table = np.zeros((2, pages - 2), np.int64)
    table[0], table[1, :2] = np.arange(pages - 2), [pages - 2, pages - 1]
    g = torch.Generator().manual_seed(long)
    rows = [torch.randn((sum(new), 2, dim), generator=g).to(BF16).cuda() for _ in range(2)]
    k, v = (torch.zeros((pages, 2, page, dim), dtype=BF16, device="cuda") for _ in range(2))
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")   # noqa: E731
    ws = pc.kv_append(pc.PagedCache(k, v), i32(table), i32(kv), i32([0, new[0], sum(new)]), *rows, max_kv=most)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 2
    for x, r in zip((k, v), rows):
        slots = x.transpose(1, 2).reshape(-1, 2, dim)
        want = torch.zeros_like(slots)
        want[most - 4:most] = r[:4]
        want[(pages - 2) * page + 18:(pages - 2) * page + 20] = r[new[0]:]
        assert torch.equal(slots, want)


@pytest.mark.parametrize("new,most", [(4, 3), (8, 1), (40, 39), (200, 130)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 50), (False, 70)])
def test_rows_past_the_bound_change_no_others(new, most, causal, window):
    """Sequences of more rows than max_q are reported; the first max_q of them, and the other
    sequences, have the positions and results that they have."""
    c = Case([500, 3000, 90], [new, new, 1], heads=8, kvh=2, seed=new)
    got = c.run(causal=causal, window=window, max_q=most)
    torch.cuda.synchronize()
    assert pc.workspace_status(got[3]) == 2
    want, tol = c.want(causal=causal, window=window)
    for first in (0, new, 2 * new):
        rows = slice(first, first + (most if first < 2 * new else 1))
        for i in range(2):
            assert np.all(np.abs(got[i][rows].cpu().double().numpy() - want[i][rows]) <= tol[i][rows])


@pytest.mark.parametrize("new", [1, 5, 40])
@pytest.mark.parametrize("kv", [200, 3000])
def test_results_in_place_and_between_queries(new, kv):
    """out over q itself, and in the gaps of q's rows, heads and [head, row] blocks."""
    c = Case([kv, 90], [new, new], heads=8, kvh=2, seed=kv + new)
    want = [x.clone() for x in c.run()[:2]]
    q, (rows, heads, dim) = c.q.clone(), c.q.shape
    empty = lambda *shape: torch.zeros(shape, dtype=c.dtype, device="cuda")   # noqa: E731
    pairs = [(x, x) for x in (q.clone(),)]
    x = empty(rows, 2 * heads, dim)
    pairs.append((x[:, :heads], x[:, heads:]))
    x = empty(rows, 2 * heads, dim)
    pairs.append((x[:, heads:], x[:, :heads]))
    x = empty(rows, heads, 2 * dim)
    pairs.append((x[..., :dim], x[..., dim:]))
    x = empty(heads, rows, 2 * dim)
    pairs.append((x[..., :dim].transpose(0, 1), x[..., dim:].transpose(0, 1)))
    x = empty(heads, 2 * rows, dim)
    pairs.append((x[:, :rows].transpose(0, 1), x[:, rows:].transpose(0, 1)))
    for src, dst in pairs:
        src.copy_(q)
        c.q = src
        got = c.run(out=dst)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.q = q
    with pytest.raises(pc.PcError):
        c.run(out=c.q, weight_out=torch.zeros((2, 2, c.cols * 16), device="cuda"))


@pytest.mark.parametrize("cache", ["same", "fp8"])
@pytest.mark.parametrize("window", [0, 300])
def test_weights_of_few_rows_with_room_for_many_slots(cache, window):
    """Above 2^30 scores of room none are kept, and results are what they are below."""
    c = Case([700, 3000, 0, 65] + [20] * 60, [4, 1, 0, 3] + [2] * 60, heads=64, kvh=8, dim=64, page=64,
             cache=FP8 if cache == "fp8" else None, weights=True, seed=11, cols=1 + (1 << 30) // (64 * 8 * 32 * 64))
    got = c.run(window=window)
    c.check(got=got, window=window)
    below = c.run(window=window, max_kv=3008, ws=got[3])
    torch.cuda.synchronize()
    for x, y in zip(got[:2], below[:2]):
        assert torch.equal(x, y)
    base = c.weight.clone()
    got = c.run(window=window, weight_out=c.weight)[2].clone()      # in place
    c.weight = base
    c.check(got=(None, None, got, below[3]), window=window)


@pytest.mark.parametrize("dim", [144, 256])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, FP8), (F16, FP8)], ids=["bf16", "f16", "bf16-fp8", "f16-fp8"])
def test_cut_sequences_of_wide_heads(dim, new, dtype, cache):
    """Parts and joins of 256 dimensions, and more than 64 groups of 16 slots in a range."""
    for heads, kvh, page in ((8, 1, 16), (4, 2, 24)):
        c = Case([5000, 300], [new, new], heads=heads, kvh=kvh, dim=dim, page=page, dtype=dtype, cache=cache, seed=dim + new,
                 weights=True)
        c.check()
        c.check(window=1700)


@pytest.mark.parametrize("n", [65, 150])
@pytest.mark.parametrize("new", [1, 12])
@pytest.mark.parametrize("page", [16, 10])
def test_cut_sequences_among_many(n, new, page):
    """More sequences than lanes of a wave, with cut ones before and behind the 64th."""
    r = np.random.default_rng(n + new)
    kv = r.integers(0, 90, n)
    for s in (0, 5, 63, 64, n - 1):
        kv[s] = r.integers(2000, 4000)
    m = np.minimum(r.integers(0, new + 1, n), kv)
    m[[0, 5, 63, 64, n - 1]] = new
    c = Case(kv, m, heads=8, kvh=2, dim=32, page=page, seed=n + new, weights=True)
    c.check()
    c.check(window=900)


@pytest.mark.parametrize("dtype,cache,dim", [(BF16, BF16, 128), (F16, F16, 96), (BF16, FP8, 80)], ids=["bf16", "f16", "fp8"])
def test_tall_tiles_of_rows(dtype, cache, dim):
    """Up to three sequences of 2,048 rows (tokens times heads of a group) for each, with room for 8,192 slots."""
    for kv, new, window in (([1300], [260], 0), ([2200, 530], [520, 300], 0), ([900, 1500, 500], [20, 770, 300], 700)):
        c = Case(kv, new, heads=8, kvh=1, dim=dim, page=16, dtype=dtype, cache=cache, weights=True, seed=dim + len(kv), cols=512)
        c.check(window=window)


def test_tall_tiles_do_not_show_what_is_masked():
    c = Case([1400], [300], heads=8, kvh=1, dim=128, page=16, seed=5, cols=512)
    for j in (1399, 1150, 1200):
        page, off = int(c.table[0, j // 16]), j % 16
        c.vc[page, 0, off, 3 + j % 7] = float("nan") if j % 2 else float("inf")
    page, off = int(c.table[0, 1390 // 16]), 1390 % 16
    c.kc[page, 0, off, 7] = float("nan")
    c.check()


@pytest.mark.parametrize("n", [12, 16])
@pytest.mark.parametrize("even", [True, False])
def test_chunks_of_even_and_uneven_rows(n, even):
    """From twelve sequences on uneven ones are cut finer, and cut ones come first."""
    r = np.random.default_rng(n)
    new = np.full(n, 40) if even else np.concatenate([[40, 0], r.integers(1, 30, n - 2)])
    kv = new + np.concatenate([r.integers(0, 200, n - 3), [3000, 0, 1500]])
    c = Case(kv, new, heads=8, kvh=2, dim=64, seed=n, weights=True)
    c.check()
    c.check(window=500)


@pytest.mark.parametrize("n_seqs", [1, 300])
@pytest.mark.parametrize("heads,dim,dtype", [(1, 16, BF16), (4, 64, F16), (5, 64, BF16)])
def test_append_of_very_many_rows(n_seqs, heads, dim, dtype):
    """From 65,536 rows on those of small 16-bit entries share waves: every slot, with empty
    sequences among the others, rows without a slot and a page that is not there."""
    r = np.random.default_rng(n_seqs + dim)
    rows, page = 65536 + 5, 10
    off = np.concatenate([[0], np.sort(r.integers(0, rows + 1, n_seqs - 1)), [rows]])
    new = np.diff(off)
    kv = np.maximum(0, new + r.integers(-3, 30, n_seqs))
    each = (kv + page - 1) // page
    pages = int(each.sum())
    table = np.full((n_seqs, int(each.max())), -1, np.int64)
    order = r.permutation(pages)
    for s, at in enumerate(np.cumsum(each) - each):
        table[s, :each[s]] = order[at:at + each[s]]
    last = int(np.argmax(new))
    table[last, each[last] // 2] = pages
    g = torch.Generator(device="cuda").manual_seed(n_seqs)
    k, v = (torch.zeros((pages, heads, page, dim), dtype=dtype, device="cuda") for _ in range(2))
    kn, vn = (torch.randn((rows, heads, dim), generator=g, device="cuda").to(dtype) for _ in range(2))
    seq = np.repeat(np.arange(n_seqs), new)
    slot = kv[seq] - off[seq + 1] + np.arange(rows)
    at = table[seq, np.maximum(slot, 0) // page]
    fine = (slot >= 0) & (at >= 0) & (at < pages)
    take, to, where = (torch.from_numpy(x[fine]).cuda() for x in (np.arange(rows), at, slot % page))
    want = [torch.zeros_like(k), torch.zeros_like(v)]
    for w, x in zip(want, (kn, vn)):
        w[to, :, where] = x[take]
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")   # noqa: E731
    ws = pc.kv_append(pc.PagedCache(k, v), i32(table), i32(kv), i32(off), kn, vn)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 2
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
