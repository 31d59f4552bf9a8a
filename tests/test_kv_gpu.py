"""pc_kv_append and pc_kv_evict against their definitions: every slot of the cache,
every kept index; types, lengths, pages, ties, values that are not finite, refusals."""
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


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int64).astype(np.int32)).cuda()


def bits(x):
    return x.view(torch.uint8 if x.element_size() == 1 else torch.int16)


def pool(pages, kvh, page, dim, dtype, g, slots_first=False):
    x = (torch.randn((pages, kvh, page, dim), generator=g) * 3).to(dtype)
    if slots_first:
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    return x.cuda()


def tables(kv, page, g, spare=2, cols=0):
    each = (np.asarray(kv) + page - 1) // page
    order = torch.randperm(int(each.sum()) + spare, generator=g).numpy()
    table = np.full((len(kv), max(1, int(each.max()), cols)), -1, np.int64)
    at = 0
    for s, n in enumerate(each):
        table[s, :n] = order[at:at + n]
        at += n
    return table, order.size


# ------------------------------------------------------------------- append

@pytest.mark.parametrize("kv,new", [([1], [1]), ([17, 0, 40, 33], [1, 0, 1, 1]), ([50, 300, 24, 7], [50, 111, 1, 0]),
                                    (list(range(1, 140)), [1 + i % 3 if i > 3 else 1 for i in range(139)])],
                         ids=["one", "decode", "chunks", "many"])
@pytest.mark.parametrize("page", [1, 16, 24, 100])
@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, FP8), (F16, FP8)],
                         ids=["bf16", "f16", "bf16-fp8", "f16-fp8"])
def test_append(kv, new, page, dtype, cache):
    g = torch.Generator().manual_seed(len(kv) + page)
    kvh, dim = 3, 48
    table, pages = tables(kv, page, g)
    k, v = (pool(pages, kvh, page, dim, cache, g, slots_first=page == 24) for _ in range(2))
    off = np.concatenate([[0], np.cumsum(new)])
    fused = (torch.randn((int(off[-1]), 2 + 2 * kvh, dim), generator=g) * 4).to(dtype).cuda()
    kn, vn = fused[:, 2:2 + kvh], fused[:, 2 + kvh:]
    scales = [(0.01 + torch.rand(kvh, generator=g)).cuda() if cache == FP8 else None for _ in range(2)]
    want = []
    for x, rows, sc in ((k, kn, scales[0]), (v, vn, scales[1])):
        y = x.detach().cpu().float().numpy().astype(np.float64)
        r = rows.cpu().float().numpy()
        if sc is not None:
            r = kv_plain.nearest_e4m3((r / sc.cpu().numpy()[None, :, None]).astype(np.float64))   # a quotient in 32 bits
        for s in range(len(kv)):
            for i in range(new[s]):
                j = kv[s] - new[s] + i
                y[table[s, j // page], :, j % page] = r[off[s] + i]
        want.append(y)
    ws = pc.kv_append(pc.PagedCache(k, v, *scales), i32(table), i32(kv), i32(off), kn, vn)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 0
    for x, y in zip((k, v), want):
        assert np.array_equal(x.cpu().float().numpy().astype(np.float64), y)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_append_rounds_to_the_nearest_code(dtype):
    """Every 16-bit pattern through an 8-bit cache: ties, subnormals, the largest value, infinities, NaN."""
    dim, page = 64, 64
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).view(1024, 1, dim).cuda()
    table, pages = tables([1024], page, torch.Generator().manual_seed(0))
    k = torch.zeros((pages, 1, page, dim), dtype=FP8, device="cuda")
    v = torch.zeros_like(k)
    scales = [torch.ones(1, device="cuda"), torch.full((1,), 0.37, device="cuda")]
    ws = pc.kv_append(pc.PagedCache(k, v, *scales), i32(table), i32([1024]), i32([0, 1024]), x, x)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 0
    for got, sc in ((k, 1.0), (v, 0.37)):
        got = got[i32(table)[0].long()].transpose(1, 2).reshape(1024, 1, dim).cpu().float().numpy().astype(np.float64)
        q = (x.cpu().float().numpy() / np.float32(sc)).astype(np.float64)
        want = kv_plain.nearest_e4m3(q)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


def test_append_leaves_out_what_does_not_fit():
    g = torch.Generator().manual_seed(1)
    page, kvh, dim = 16, 2, 32
    kv, new = [40, 20, 3], [3, 2, 5]                 # the last chunk has two rows before its first slot
    table, pages = tables([40, 20, 5], page, g)

    def run(change):
        k, v = (torch.zeros((pages, kvh, page, dim), dtype=BF16, device="cuda") for _ in range(2))
        a = dict(table=i32(table), kv=i32(kv), off=i32([0, 3, 5, 10]))
        change(a)
        rows = torch.ones((10, kvh, dim), dtype=BF16, device="cuda")
        ws = pc.kv_append(pc.PagedCache(k, v), a["table"], a["kv"], a["off"], rows, rows)
        torch.cuda.synchronize()
        assert torch.equal(k, v)
        return pc.workspace_status(ws), int(k[:, 0, :, 0].sum().item())
    assert run(lambda a: None) == (2, 8)
    assert run(lambda a: a["kv"].copy_(i32([40, 20, 5]))) == (0, 10)
    assert run(lambda a: a["table"][0].fill_(pages)) == (2, 5)
    assert run(lambda a: a["table"][1].fill_(-1)) == (2, 6)
    assert run(lambda a: a["kv"].copy_(i32([4000, 20, 5])))[0] == 2
    assert run(lambda a: a["off"].copy_(i32([0, 3, 2, 10])))[0] == 2
    assert run(lambda a: a["off"].copy_(i32([0, 3, 5, 11])))[0] == 2
    assert run(lambda a: a["off"].copy_(i32([2, 3, 5, 10])))[0] == 2


def test_append_nothing_and_many_pages():
    g = torch.Generator().manual_seed(2)
    k, v = (torch.zeros((70, 1, 2, 16), dtype=F16, device="cuda") for _ in range(2))
    none = torch.empty((0, 1, 16), dtype=F16, device="cuda")
    ws = pc.kv_append(pc.PagedCache(k, v), i32([[0], [0]]), i32([2, 0]), i32([0, 0, 0]), none, none)
    assert pc.workspace_status(ws) == 0
    kv = [1, 130, 5]                                  # 65 pages of one sequence among short ones
    table, pages = tables(kv, 2, g)
    rows = torch.randn((136, 1, 16), generator=g).to(F16).cuda()
    k, v = (torch.zeros((pages, 1, 2, 16), dtype=F16, device="cuda") for _ in range(2))
    ws = pc.kv_append(pc.PagedCache(k, v), i32(table), i32(kv), i32([0, 1, 131, 136]), rows, rows)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 0
    got = k[i32(table)[1].long()].transpose(1, 2).reshape(-1, 1, 16)
    assert torch.equal(got, rows[1:131])
    bad = i32(table)
    bad[1, 64] = pages
    ws = pc.kv_append(pc.PagedCache(k, v), bad, i32(kv), i32([0, 1, 131, 136]), rows, rows)
    assert pc.workspace_status(ws) == 2


def test_append_refusals():
    k = torch.zeros((4, 2, 16, 32), dtype=BF16, device="cuda")
    cache = pc.PagedCache(k, k.clone())
    rows = torch.zeros((3, 2, 32), dtype=BF16, device="cuda")
    ok = dict(cache=cache, page_table=i32([[0, 1]]), kv_len=i32([9]), q_off=i32([0, 3]), k=rows, v=rows)
    pc.kv_append(**ok)

    def refused(**kw):
        with pytest.raises(pc.PcError):
            pc.kv_append(**dict(ok, **kw))
    refused(k=rows.to(F16), v=rows.to(F16))
    refused(v=rows[:2])
    refused(k=rows[:, :1], v=rows[:, :1])
    refused(k=torch.zeros((3, 2, 36), dtype=BF16, device="cuda")[..., 4:], v=rows)
    refused(q_off=i32([0, 1, 3]))
    refused(max_kv=33)
    refused(kv_len=torch.tensor([9], device="cuda"))
    refused(ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    odd = torch.zeros((4, 2, 16, 40), dtype=BF16, device="cuda")
    refused(cache=pc.PagedCache(odd, odd.clone()), k=torch.zeros((3, 2, 40), dtype=BF16, device="cuda"),
            v=torch.zeros((3, 2, 40), dtype=BF16, device="cuda"))     # head_dim is no multiple of 16


# -------------------------------------------------------------------- evict

def weights(kind, shape, g):
    if kind == "random":
        return torch.randn(shape, generator=g).exp()
    if kind == "ties":
        return torch.randint(0, 4, shape, generator=g).float() / 2
    if kind == "zeros":
        return torch.zeros(shape)
    if kind == "close":      # keys that differ in their last bits only
        return (torch.randint(0, 300, shape, generator=g) + 0x3F800000).to(torch.int32).view(torch.float32)
    w = torch.randn(shape, generator=g)
    odd = torch.tensor([float("nan"), float("inf"), float("-inf"), 0.0, -0.0, 1e-42, -1e-42, -float("nan")])
    pick = torch.randint(0, 16, shape, generator=g)
    return torch.where(pick < 8, odd[pick.clamp(max=7)], w)


@pytest.mark.parametrize("kind", ["random", "ties", "zeros", "close", "odd"])
@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (20, 5), (64, 64), (700, 0), (1500, 100), (5000, 10)])
@pytest.mark.parametrize("dtype", [BF16, FP8], ids=["bf16", "fp8"])
def test_evict(kind, budget, recent, dtype):
    g = torch.Generator().manual_seed(budget + recent)
    kv = np.array([0, 1, 19, 64, 65, 1023, 1500, 4100])
    page, kvh, dim = 24, 2, 32
    table, pages = tables(kv, page, g)
    keep = min(budget, int(kv.max()))
    cols = (budget + page - 1) // page
    dst = torch.randperm(len(kv) * cols, generator=g).numpy().reshape(len(kv), cols) + pages
    total = pages + dst.size
    k, v = (pool(total, kvh, page, dim, dtype, g) for _ in range(2))
    scales = [torch.ones(kvh, device="cuda") if dtype == FP8 else None] * 2
    w = weights(kind, (len(kv), kvh, int(kv.max()) + 3), g)
    before = [bits(x).cpu().numpy().copy() for x in (k, v)]
    got = pc.kv_evict(pc.PagedCache(k, v, *scales), i32(table), i32(kv), w.cuda(), budget, recent, dst_table=i32(dst))
    torch.cuda.synchronize()
    assert pc.workspace_status(got["ws"]) == 0
    kept, moved, new_len = kv_plain.evict(w.numpy(), kv, budget, recent)
    assert np.array_equal(got["new_len"].cpu().numpy(), new_len) and keep == new_len.max()
    assert np.array_equal(got["kept"].cpu().numpy(), kept)
    assert np.array_equal(got["weight"].cpu().numpy().view(np.int32)[~np.isnan(moved)], moved.view(np.int32)[~np.isnan(moved)])
    assert np.array_equal(np.isnan(got["weight"].cpu().numpy()), np.isnan(moved))
    for x, b in zip((k, v), before):
        for s in range(len(kv)):
            for h in range(kvh):
                n = int(new_len[s])
                j, r = kept[s, h, :n], np.arange(n)
                b[dst[s, r // page], h, r % page] = b[table[s, j // page], h, j % page]
        assert np.array_equal(bits(x).cpu().numpy(), b)


@pytest.mark.parametrize("length", [1, 1024, 1025, 8191, 40000, 131072, 300001])
def test_evict_long(length):
    """Against a stable sort, at lengths on either side of what one workgroup holds."""
    g = torch.Generator().manual_seed(length)
    kv = np.array([length, max(1, length // 3)])
    w = (torch.randn((2, 3, length), generator=g) * 2).exp()
    w = torch.where(torch.rand(w.shape, generator=g) < 0.3, (w * 4).round() / 4, w)
    cache = pc.PagedCache(*(torch.zeros((1, 3, 16, 16), dtype=BF16, device="cuda") for _ in range(2)))
    table = torch.zeros((2, (length + 15) // 16), dtype=torch.int32, device="cuda")
    for budget, recent in ((1, 0), (max(1, length // 7), length // 50), (max(1, length - 1), 0), (length, 1)):
        got = pc.kv_evict(cache, table, i32(kv), w.cuda(), budget, recent)
        torch.cuda.synchronize()
        assert pc.workspace_status(got["ws"]) == 0
        for s in range(2):
            n = int(kv[s])
            m = min(n, budget)
            late = min(recent, m)
            order = torch.sort(w[s, :, :n - late], dim=-1, descending=True, stable=True).indices[:, :m - late]
            want = torch.cat([order.sort(-1).values, torch.arange(n - late, n).expand(3, late)], 1)
            assert torch.equal(got["kept"][s, :, :m].cpu().long(), want)
            assert bool((got["kept"][s, :, m:] == -1).all()) and bool((got["weight"][s, :, m:] == 0).all())
            assert torch.equal(got["weight"][s, :, :m].cpu(), w[s].gather(1, want))


def test_evict_bad_layouts_and_shared_pages():
    g = torch.Generator().manual_seed(3)
    page, kvh, dim, kv = 16, 2, 32, [60, 60]
    k, v = (pool(20, kvh, page, dim, BF16, g) for _ in range(2))
    cache = pc.PagedCache(k, v)
    w = torch.rand((2, kvh, 60), generator=g).cuda()
    table = i32([[0, 1, 2, 3], [0, 1, 2, 4]])          # a shared prefix of three pages
    dst = i32([[10, 11], [12, 13]])
    before = k.clone()
    got = pc.kv_evict(cache, table, i32(kv), w, 30, 4, dst_table=dst)
    torch.cuda.synchronize()
    assert pc.workspace_status(got["ws"]) == 0 and torch.equal(k[:10], before[:10]) and torch.equal(k[14:], before[14:])
    assert pc.workspace_status(pc.kv_evict(cache, table, i32([60, 64 * 16]), w, 30, 4, dst_table=dst)["ws"]) == 2
    for t, d in ((i32([[0, 1, 2, 20], [0, 1, 2, 4]]), dst), (table, i32([[10, 11], [12, -1]]))):
        before = k.clone()
        got = pc.kv_evict(cache, t, i32(kv), w, 30, 4, dst_table=d)
        torch.cuda.synchronize()
        assert pc.workspace_status(got["ws"]) == 2 and torch.equal(k[:10], before[:10]) and torch.equal(k[14:], before[14:])


def test_evict_refusals():
    k = torch.zeros((4, 2, 16, 32), dtype=BF16, device="cuda")
    cache = pc.PagedCache(k, k.clone())
    ok = dict(cache=cache, page_table=i32([[0, 1]]), kv_len=i32([9]), weight=torch.zeros((1, 2, 32), device="cuda"),
              budget=4, recent=1)
    pc.kv_evict(**ok)

    def refused(**kw):
        with pytest.raises(pc.PcError):
            pc.kv_evict(**dict(ok, **kw))
    refused(budget=0)
    refused(recent=5)
    refused(weight=torch.zeros((1, 3, 32), device="cuda"))
    refused(weight=torch.zeros((1, 2, 32), device="cuda", dtype=torch.float64))
    refused(max_kv=40)
    refused(dst_table=i32([[2]]), budget=17)
    refused(ws=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_append_and_evict_replay_in_a_graph():
    g = torch.Generator().manual_seed(4)
    page, kvh, dim = 16, 2, 64
    kv, new = [200, 90], [3, 1]
    table, pages = tables(kv, page, g)
    dst = np.arange(8).reshape(2, 4) + pages
    base = [pool(pages + 8, kvh, page, dim, BF16, g) for _ in range(2)]
    k, v = (x.clone() for x in base)
    cache = pc.PagedCache(k, v)
    rows = torch.randn((4, kvh, dim), generator=g).to(BF16).cuda()
    w = torch.rand((2, kvh, 208), generator=g).cuda()
    a = dict(t=i32(table), kv=i32(kv), off=i32([0, 3, 4]), dst=i32(dst))
    ws = pc.workspace(256)

    def step(out=None):
        pc.kv_append(cache, a["t"], a["kv"], a["off"], rows, rows, ws=ws)
        return pc.kv_evict(cache, a["t"], a["kv"], w, 60, 5, dst_table=a["dst"], out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        w.copy_(torch.rand((2, kvh, 208), generator=g))
        rows.copy_(torch.randn((4, kvh, dim), generator=g).to(BF16))
        for x, y in zip((k, v), base):
            x.copy_(y)
        eager = step()
        want = [x.clone() for x in (k, v, eager["kept"], eager["weight"])]
        for x, y in zip((k, v), base):
            x.copy_(y)
        out["kept"].fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((k, v, out["kept"], out["weight"]), want))


@pytest.mark.parametrize("length", [8192, 8193, 16384, 16385, 32769, 70000])
@pytest.mark.parametrize("kind", ["zeros", "ties", "odd"])
def test_evict_ties_over_segments(length, kind):
    """Long rows are selected in segments; equal weights go to the lowest slots over all of them."""
    g = torch.Generator().manual_seed(length)
    kv = np.array([length, length - 5000, 3, 0])
    w = weights(kind, (4, 2, length), g)
    cache = pc.PagedCache(*(torch.zeros((1, 2, 64, 16), dtype=BF16, device="cuda") for _ in range(2)))
    table = torch.zeros((4, (length + 63) // 64), dtype=torch.int32, device="cuda")
    for budget, recent in ((length // 3, 7), (length - 5000, 100), (length, 0)):
        got = pc.kv_evict(cache, table, i32(kv), w.cuda(), budget, recent)
        torch.cuda.synchronize()
        assert pc.workspace_status(got["ws"]) == 0
        kept, moved, new_len = kv_plain.evict(w.numpy(), kv, budget, recent)
        assert np.array_equal(got["new_len"].cpu().numpy(), new_len)
        assert np.array_equal(got["kept"].cpu().numpy(), kept)
        nan = np.isnan(moved)
        assert np.array_equal(np.isnan(got["weight"].cpu().numpy()), nan)
        assert np.array_equal(got["weight"].cpu().numpy()[~nan], moved[~nan])


@pytest.mark.parametrize("n_seqs", [1, 3, 70, 5000])
@pytest.mark.parametrize("cache,heads,dim", [(BF16, 3, 80), (FP8, 4, 128), (FP8, 1, 16)])
def test_append_many_rows(n_seqs, cache, heads, dim):
    """Above 8,192 rows, in sequences of any length, many of them empty; rows without a slot or
    a page are left out."""
    r = np.random.default_rng(n_seqs + dim)
    rows, page = 9001, 24
    cut = np.sort(r.integers(0, rows + 1, n_seqs - 1))
    off = np.concatenate([[0], cut, [rows]])
    new = np.diff(off)
    kv = new + r.integers(0, 30, n_seqs)
    g = torch.Generator().manual_seed(n_seqs)
    table, pages = tables(kv, page, g)
    lost = 0
    if n_seqs == 3:
        kv[1] = max(0, new[1] - 5)                    # its first rows have no slot
        table[2, 1] = pages + 7                       # no page
    k, v = (pool(pages, heads, page, dim, cache, g) for _ in range(2))
    kn, vn = ((torch.randn((rows, heads, dim), generator=g) * 3).to(BF16).cuda() for _ in range(2))
    scales = [torch.full((heads,), 0.5, device="cuda") if cache == FP8 else None for _ in range(2)]
    want = []
    for x, n in ((k, kn), (v, vn)):
        y = x.detach().cpu().float().numpy().astype(np.float64)
        z = n.cpu().float().numpy().astype(np.float64)
        if cache == FP8:
            z = kv_plain.nearest_e4m3(z / 0.5)
        for s in range(n_seqs):
            for i in range(new[s]):
                j = kv[s] - new[s] + i
                if j < 0 or table[s, j // page] >= pages:
                    lost += 1
                    continue
                y[table[s, j // page], :, j % page] = z[off[s] + i]
        want.append(y)
    ws = pc.kv_append(pc.PagedCache(k, v, *scales), i32(table), i32(kv), i32(off), kn, vn)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == (2 if lost else 0) and (lost > 0) == (n_seqs == 3)
    for x, y in zip((k, v), want):
        assert np.array_equal(x.cpu().float().numpy().astype(np.float64), y)
