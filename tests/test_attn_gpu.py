"""pc_attn_paged against the definition in 64 bits: types, head layouts, lengths from
none to long, pages of any size, masks, strides, streams, graphs, refusals."""
import numpy as np
import pytest
import torch

import kv_plain
from paper_2609_28870_amd import pc

pytestmark = pytest.mark.gpu
BF16, F16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class Case:
    """A cache with shuffled pages whose unused slots and pages hold NaN, and a chunk."""

    def __init__(self, kv, new, heads=8, kvh=2, dim=64, page=16, dtype=BF16, cache=None, seed=0, slots_first=False,
                 spare_pages=3, weights=False, cols=0):
        g = torch.Generator().manual_seed(seed)
        kv_np, new_np = np.array(kv, np.int64), np.array(new, np.int64)
        self.kv, self.new, self.dtype, self.page = kv_np, new_np, dtype, page
        cache = cache or dtype
        n = len(kv)
        each = (kv_np + page - 1) // page
        pages = int(each.sum()) + spare_pages
        order = torch.randperm(pages, generator=g).numpy()
        self.cols = max(1, int(each.max()) if n else 1, cols)
        self.table = np.full((n, self.cols), 0x7FFFFFFF, np.int64)     # entries past the length name no page
        at = 0
        x = torch.randn((2, pages, kvh, page, dim), generator=g)
        used = torch.zeros((pages, page), dtype=torch.bool)
        for s in range(n):
            self.table[s, :each[s]] = order[at:at + each[s]]
            for p in range(int(each[s])):
                used[order[at + p], :min(page, int(kv_np[s]) - p * page)] = True
            at += int(each[s])
        self.ks = self.vs = None
        if cache == FP8:
            self.ks, self.vs = (0.01 + 0.02 * torch.rand(kvh, generator=g)).cuda(), (0.01 + 0.02 * torch.rand(kvh, generator=g)).cuda()
            x = (x * 60).clamp(-448, 448)
        x = x.masked_fill(~used[None, :, None, :, None], float("nan")).to(cache)
        if slots_first:
            kc, vc = (x[i].transpose(1, 2).contiguous().cuda().transpose(1, 2) for i in range(2))
        else:
            kc, vc = x[0].cuda(), x[1].cuda()
        self.kc, self.vc = kc, vc
        self.q_off = np.concatenate([[0], np.cumsum(new_np)])
        self.q = torch.randn((int(self.q_off[-1]), heads, dim), generator=g).to(dtype).cuda()
        self.weight = torch.rand((n, kvh, self.cols * page), generator=g).cuda() if weights else None
        self.d_table = torch.from_numpy(self.table.astype(np.int32)).cuda()
        self.d_kv = torch.from_numpy(kv_np.astype(np.int32)).cuda()
        self.d_off = torch.from_numpy(self.q_off.astype(np.int32)).cuda()

    def run(self, causal=True, window=0, scale=None, **kw):
        cache = pc.PagedCache(self.kc, self.vc, self.ks, self.vs)
        kw.setdefault("max_q", int(self.new.max()) if len(self.new) else 0)
        kw.setdefault("want_lse", True)
        return pc.attn_paged(self.q, cache, self.d_table, self.d_kv, self.d_off, causal=causal, window=window, scale=scale,
                             weight=self.weight, **kw)

    def want(self, causal=True, window=0, scale=None):
        k, v = kv_plain.cache_values(self.kc, self.vc, self.ks, self.vs)
        scale = self.q.shape[2] ** -0.5 if scale is None else float(np.float32(scale))
        return kv_plain.attention(self.q, k, v, self.table, self.kv, self.q_off, scale, causal, window, self.weight, self.dtype)

    def check(self, got=None, **kw):
        if got is None:
            got = self.run(**kw)
        torch.cuda.synchronize()
        assert pc.workspace_status(got[3]) == 0
        want, tol = self.want(**kw)
        for name, x, y, t in zip(("out", "lse", "weight"), got, want, tol):
            if x is None or y is None:
                continue
            x = x.detach().cpu().double().numpy()
            fine = np.isfinite(y)
            assert np.array_equal(np.isfinite(x), fine), name
            assert np.array_equal(x[~fine & ~np.isnan(y)], y[~fine & ~np.isnan(y)]), name
            assert np.array_equal(np.isnan(x), np.isnan(y)), name
            over = np.abs(x[fine] - y[fine]) - t[fine]
            assert over.size == 0 or over.max() <= 0, (name, float(over.max()))


LENGTHS = {
    "one": ([1], [1]),
    "decode": ([1, 33, 200, 0, 64, 65], [1, 1, 1, 0, 1, 1]),
    "few": ([7, 40, 300, 129], [3, 4, 1, 0]),
    "chunks": ([70, 0, 5, 260, 128], [70, 0, 5, 41, 9]),
    "empty_rows": ([3, 0, 20], [9, 4, 20]),          # rows before the first slot see nothing
    "long": ([3001], [1]),
    "long_chunk": ([2100, 90], [150, 33]),
}


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("cache", ["same", "fp8"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_lengths_and_types(lengths, dtype, cache):
    kv, new = LENGTHS[lengths]
    c = Case(kv, new, dtype=dtype, cache=FP8 if cache == "fp8" else None, seed=len(lengths), weights=True)
    if lengths == "empty_rows":
        # such a chunk is reported; what its rows see is still defined
        got = c.run()
        torch.cuda.synchronize()
        assert pc.workspace_status(got[3]) == 2
        want, tol = c.want()
        out, lse = got[0].cpu().double().numpy(), got[1].cpu().double().numpy()
        assert np.all(np.abs(out - want[0]) <= tol[0])
        assert np.array_equal(np.isinf(lse), np.isinf(want[1])) and np.isinf(lse).sum() == 8 * (6 + 4)
        assert np.all(out[np.isinf(lse)] == 0)
        w = got[2].cpu().double().numpy()
        assert np.all(np.abs(w - want[2]) <= tol[2])
        return
    c.check()


@pytest.mark.parametrize("heads,kvh", [(1, 1), (3, 3), (4, 1), (14, 2), (16, 2), (33, 1), (40, 1), (6, 3)])
@pytest.mark.parametrize("new", [1, 5, 40])
def test_head_groups(heads, kvh, new):
    Case([new + 100, new, new + 3], [new, new, 1], heads=heads, kvh=kvh, seed=heads + new, weights=True).check()


@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 176, 240, 256])
@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("cache", ["same", "fp8"])
def test_head_dims(dim, new, cache):
    Case([170, 50], [new, new], heads=6, kvh=2, dim=dim, dtype=F16 if dim % 32 else BF16, cache=FP8 if cache == "fp8" else None,
         seed=dim, weights=True).check()


@pytest.mark.parametrize("page", [1, 2, 5, 16, 24, 64, 100, 256, 1000])
@pytest.mark.parametrize("new", [1, 37])
def test_page_sizes(page, new):
    Case([311, 64, 63, new + 1], [new] * 4, page=page, seed=page, weights=True).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 7, 64, 100, 5000, 2 ** 32 - 1])
@pytest.mark.parametrize("new", [1, 4, 50])
def test_masks(causal, window, new):
    Case([300, 64, new + 33], [new] * 3, heads=8, kvh=1, page=24, seed=window % 97 + new, weights=True).check(causal=causal, window=window)


@pytest.mark.parametrize("n", [64, 65, 150])
@pytest.mark.parametrize("new", [1, 12])
def test_many_sequences(n, new):
    r = np.random.default_rng(n)
    kv = r.integers(0, 90, n)
    m = np.minimum(r.integers(0, new + 1, n), kv)
    Case(kv, m, heads=4, kvh=2, dim=32, seed=n, weights=True).check()


@pytest.mark.parametrize("new", [1, 3, 100])
@pytest.mark.parametrize("cache", ["same", "fp8"])
def test_keys_split_over_workgroups(new, cache):
    c = Case([9000, 257, 2000], [new] * 3, heads=8, kvh=1, dim=128, page=64, cache=FP8 if cache == "fp8" else None, seed=5, weights=True)
    c.check()
    c.check(window=700)


@pytest.mark.parametrize("new", [1, 40])
def test_strides(new):
    """Pages as [page, slot, head, dim], queries and results inside wider rows."""
    c = Case([100, 41], [new, new], slots_first=True, weights=True, seed=9)
    rows, heads, dim = c.q.shape
    wide = torch.randn(rows, heads + 4, dim, device="cuda").to(c.dtype)
    wide[:, 2:2 + heads] = c.q
    c.q = wide[:, 2:2 + heads]
    res = torch.full((heads, rows, dim + 8), 7.0, dtype=c.dtype, device="cuda")
    out = res[:, :, :dim].transpose(0, 1)
    got = c.run(out=out)
    c.check(got=got)
    assert bool((res[:, :, dim:] == 7).all())


@pytest.mark.parametrize("new", [1, 40])
def test_scales(new):
    for scale in (-0.3, 0.0, 1e-20, 2.0):
        Case([100, 41], [new, new], weights=True, seed=3).check(scale=scale)
    c = Case([100, 41], [new, new], cache=FP8, weights=True, seed=4)
    c.ks[0], c.ks[1], c.vs[0] = 0.0, -0.02, -0.5
    c.check()


@pytest.mark.parametrize("new", [4, 64])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("cache", ["same", "fp8"])
def test_what_a_row_does_not_see_stays_out(new, dtype, cache):
    """Keys and values that are not finite, at slots that some rows of the chunk see."""
    c = Case([90, 70], [new, new], heads=4, kvh=2, dtype=dtype, cache=FP8 if cache == "fp8" else None, page=16, seed=2)
    n = 90
    bad = [n - 1, n - 2] + ([n - new + 7] if new > 8 else [])
    for i, j in enumerate(bad):
        page, off = int(c.table[0, j // 16]), j % 16
        if cache == "fp8":
            c.vc[page, :, off].view(torch.uint8)[:, 3 + i] = 0x7F
        else:
            c.vc[page, 0, off, 5 + i] = float("inf") if i else float("nan")
            c.vc[page, 1, off, 40] = float("-inf")
    page, off = int(c.table[0, (n - 3) // 16]), (n - 3) % 16
    if cache == "fp8":
        c.kc[page, 1, off].view(torch.uint8)[7] = 0xFF
    else:
        c.kc[page, 1, off, 7] = float("nan")
    got = c.run()
    c.check(got=got)
    out = got[0][:new].cpu()
    seen = [j for j in bad + [n - 3] if j <= n - new]
    assert not seen or new > 8
    first = out[0]
    assert bool(torch.isfinite(first).all())
    assert not bool(torch.isfinite(out[new - 1]).all())


def test_a_query_that_is_not_finite_spoils_its_row_only():
    for new in (4, 64):
        c = Case([90], [new], heads=4, kvh=2, seed=8)
        ref = c.run()[0].clone()
        c.q[1, 2, 3] = float("nan")
        got = c.run()[0]
        assert bool(torch.isnan(got[1, 2]).all())
        got[1, 2] = ref[1, 2]
        assert torch.equal(got, ref)


@pytest.mark.parametrize("new", [1, 40])
def test_weights_accumulate_in_place_and_from_nothing(new):
    c = Case([100, 41, 0], [new, new, 0], weights=True, seed=12)
    base = c.weight.clone()
    ref = c.run()[2].clone()
    c.run(weight_out=c.weight)
    torch.cuda.synchronize()
    assert torch.equal(c.weight, ref)
    c.weight = None
    zero = torch.full_like(base, 9.0)
    got = c.run(weight_out=zero)[2]
    c.weight = torch.zeros_like(base)
    assert torch.equal(got, c.run()[2])
    assert bool((got[2] == 0).all()) and bool((got[0, :, 100:] == 0).all())


def test_results_repeat():
    for kv, new in (([9000, 300], [2, 2]), ([3000, 300], [300, 100])):
        c = Case(kv, new, heads=16, kvh=2, dim=128, weights=True, seed=1)
        a = [x.clone() for x in c.run()[:3]]
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(a, c.run()[:3]))


def test_other_streams():
    """Two calls on two streams, each behind the copy that brings its queries."""
    c = Case([500, 300], [40, 3], weights=True, seed=6)
    d = Case([900, 20], [1, 1], weights=True, seed=7)
    want = [c.run()[0].clone(), d.run()[0].clone()]
    host = [c.q.cpu(), d.q.cpu()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for x, s, h in ((c, streams[0], host[0]), (d, streams[1], host[1])):
        with torch.cuda.stream(s):
            x.q = torch.zeros_like(x.q)
            x.q.copy_(h)
            got.append(x.run()[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("new", [1, 40])
def test_graph(new):
    """Captured once, replayed over other queries, lengths and tables of the same bounds."""
    c = Case([500, 300, 77], [new] * 3, weights=True, seed=6)
    d = Case([120, 500, 300], [new] * 3, weights=True, seed=16)
    pages = max(c.kc.shape[0], d.kc.shape[0])
    for x in (c, d):   # one cache size for both
        pad = torch.zeros((pages - x.kc.shape[0],) + x.kc.shape[1:], dtype=x.kc.dtype, device="cuda")
        x.kc, x.vc = torch.cat([x.kc, pad]), torch.cat([x.vc, pad])
        x.weight = x.weight[:, :, :512].contiguous()
    ref = [[y.clone() for y in x.run(max_kv=512)[:3]] for x in (c, d)]
    names = ("kc", "vc", "q", "d_table", "d_kv", "d_off", "weight")
    data = [{n: getattr(x, n).clone() for n in names} for x in (c, d)]
    static = {n: data[0][n].clone() for n in names}
    for n in names:
        setattr(c, n, static[n])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = c.run(max_kv=512)
    torch.cuda.current_stream().wait_stream(side)
    out, lse, w, ws = (torch.zeros_like(x) for x in first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(max_kv=512, out=out, lse=lse, weight_out=w, ws=ws)
    for i in (0, 1, 1, 0, 1):
        for n in names:
            static[n].copy_(data[i][n])
        for y in (out, lse, w):
            y.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, w), ref[i]))
        assert pc.workspace_status(ws) == 0


def test_cache_past_32_bits():
    """Pages whose offsets pass 2^32 bytes, and 2^31 elements."""
    page, kvh, dim = 64, 4, 128
    pages = (1 << 32) // (page * kvh * dim * 2) + 40
    kc = torch.zeros((pages, kvh, page, dim), dtype=BF16, device="cuda")
    vc = torch.zeros_like(kc)
    c = Case([300, 64 * 20], [5, 40], heads=8, kvh=kvh, dim=dim, page=page, weights=True, seed=2)
    n = c.kc.shape[0]
    kc[-n:], vc[-n:] = c.kc, c.vc
    ref = [x.clone() for x in c.run()[:3]]
    c.kc, c.vc = kc, vc
    c.d_table = torch.where(c.d_table < n, c.d_table + (pages - n), c.d_table)
    got = c.run()
    assert pc.workspace_status(got[3]) == 0
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


@pytest.mark.parametrize("new", [1, 40])
def test_bad_layouts_are_reported(new):
    def status(change, **kw):
        c = Case([200, 100], [new, new], weights=True, seed=3)
        c.kw = dict(kw)
        change(c)
        got = c.run(**c.kw)
        torch.cuda.synchronize()
        return pc.workspace_status(got[3])

    def page(value):
        def change(c):
            c.d_table[1, 2] = value
        return change

    def lens(values):
        def change(c):
            c.d_kv.copy_(torch.tensor(values, dtype=torch.int32))
        return change

    def offs(values):
        def change(c):
            c.d_off.copy_(torch.tensor(values, dtype=torch.int32))
        return change
    assert status(lambda c: None) == 0
    assert status(page(-1)) == 2
    assert status(page(10 ** 6)) == 2
    assert status(lens([200, 10 ** 6])) == 2
    assert status(lens([-1, 100])) == 2
    assert status(offs([0, 2 * new + 5, 2 * new])) == 2
    assert status(offs([0, new, 2 * new + 7])) == 2
    assert status(offs([1, new, 2 * new])) == 2
    assert status(offs([0, -5, 2 * new])) == 2
    if new > 1:
        assert status(lambda c: None, max_q=new - 1) == 2


def test_nothing_to_do():
    c = Case([5, 0], [0, 0], weights=True)
    got = c.run()
    torch.cuda.synchronize()
    assert got[0].shape[0] == 0 and pc.workspace_status(got[3]) == 0
    assert torch.equal(got[2][0, :, :5], c.weight[0, :, :5]) and bool((got[2][:, :, 5:] == 0).all())
    assert bool((got[2][1] == 0).all())


def test_refusals():
    c = Case([100, 41], [4, 4], heads=8, kvh=2)
    cache = pc.PagedCache(c.kc, c.vc)
    ok = dict(q=c.q, cache=cache, page_table=c.d_table, kv_len=c.d_kv, q_off=c.d_off, max_q=4)

    def refused(**kw):
        with pytest.raises(pc.PcError):
            pc.attn_paged(**dict(ok, **kw))
    refused(q=c.q.to(F16))                                   # not the cache's type
    refused(q=c.q.float())
    refused(q=c.q[:, :7])                                    # heads do not share evenly
    refused(q=c.q[..., :48])
    refused(q=c.q.cpu())
    refused(q=c.q.transpose(1, 2).contiguous().transpose(1, 2))   # last dimension not contiguous
    wide = torch.zeros(8, 8, 68, dtype=BF16, device="cuda")
    refused(q=wide[:, :, 2:66])                              # rows not at multiples of 16 bytes
    refused(max_kv=c.cols * 16 + 1)
    refused(scale=float("nan"))
    refused(scale=float("inf"))
    refused(q_off=c.d_off[:2])
    refused(q_off=c.d_off.long())
    refused(weight=torch.zeros(2, 2, 8, device="cuda"))
    refused(weight=torch.zeros(2, 3, 256, device="cuda"))
    refused(out=torch.zeros(8, 8, 64, dtype=F16, device="cuda"))
    refused(ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    refused(max_q=0)
    with pytest.raises(pc.PcError):
        pc.PagedCache(c.kc, c.vc, torch.ones(2, device="cuda"), None)
        pc.attn_paged(**dict(ok, cache=pc.PagedCache(c.kc, c.vc, torch.ones(2, device="cuda"), None)))
    with pytest.raises(pc.PcError):
        pc.PagedCache(c.kc, c.vc[:, :1])
    with pytest.raises(pc.PcError):
        pc.PagedCache(c.kc.float(), c.vc.float())


def test_negative_bounds_are_refused():
    c = Case([100, 41], [4, 4], heads=8, kvh=2)
    for kw in (dict(window=-1), dict(max_q=-1), dict(max_kv=-1)):
        with pytest.raises(pc.PcError):
            c.run(**kw)
    cache = pc.PagedCache(c.kc, c.vc)
    w = torch.zeros(2, 2, 112, device="cuda")
    for budget, recent in ((-1, 0), (8, -1), (8, 9), (0, 0)):
        with pytest.raises(pc.PcError):
            pc.kv_evict(cache, c.d_table, c.d_kv, w, budget, recent)


def test_decreasing_lengths_and_many_parts():
    """Sequences that are cut into ranges among ones that are not, more parts than a join takes at once."""
    kv = [40, 6000, 10, 3000, 0, 700, 5000]
    for new in (1, 2, 45):
        c = Case(kv, [min(new, n) for n in kv], heads=4, kvh=1, dim=128, page=64, weights=True, seed=new)
        c.check()
        c.check(window=1000)


@pytest.mark.parametrize("scale", [-0.2, 0.0])
@pytest.mark.parametrize("cache", ["same", "fp8"])
def test_weights_of_chunks_with_other_scales(scale, cache):
    for dim in (80, 128):
        Case([400, 300], [130, 65], heads=6, kvh=2, dim=dim, cache=FP8 if cache == "fp8" else None, weights=True, seed=dim).check(scale=scale, window=90)


@pytest.mark.parametrize("dim,page", [(80, 24), (96, 16), (128, 16), (128, 10)])
@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, FP8)], ids=["bf16", "f16", "fp8"])
def test_few_sequences_of_many_rows(dim, page, dtype, cache):
    """From 1,024 rows (tokens times heads of a group) on, with room for 8,192 slots, tiles of rows
    are twice as tall."""
    for kv, new, window in (([1300, 9], [150, 9], 0), ([150], [150], 0), ([2100, 140, 700], [129, 140, 1], 300)):
        c = Case(kv, new, heads=16, kvh=2, dim=dim, page=page, dtype=dtype, cache=cache, weights=True, seed=dim + page,
                 cols=8192 // page + 1)
        c.check(window=window)
    c.check(causal=False)


def test_many_rows_do_not_see_what_is_masked():
    c = Case([400], [160], heads=8, kvh=1, dim=128, page=16, seed=5, cols=512)
    for j in (399, 250, 300):
        page, off = int(c.table[0, j // 16]), j % 16
        c.vc[page, 0, off, 3 + j % 7] = float("nan") if j % 2 else float("inf")
    page, off = int(c.table[0, 390 // 16]), 390 % 16
    c.kc[page, 0, off, 7] = float("nan")
    c.check()
