"""pc_attn_paged and pc_kv_evict over a cache in 4 bits, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import kv_plain
import turn_plain
from paper_2609_28870_amd import pc
from test_attn_gpu import LENGTHS, Case
from test_kv_gpu import i32, tables, weights

pytestmark = pytest.mark.gpu
BF16, F16, FP4 = torch.bfloat16, torch.float16, torch.float4_e2m1fn_x2


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class Case4(Case):
    """The same pages as 4-bit codes: unused slots and pages hold codes of any value and scales of NaN."""

    def __init__(self, kv, new, slots_first=False, pad=0, seed=0, **kw):
        super().__init__(kv, new, seed=seed, **kw)
        g = torch.Generator().manual_seed(seed + 1)
        self.codes, self.exps = [], []
        for x in (self.kc, self.vc):
            y = x.cpu().float().double().numpy()
            unused = np.isnan(y).any(-1)
            codes, e = turn_plain.pack_fp4(np.nan_to_num(y), self.dtype)
            some = torch.from_numpy(unused)
            codes = torch.where(some[..., None], torch.randint(0, 256, codes.shape, generator=g).to(torch.uint8), codes)
            e = torch.where(some[..., None], torch.full_like(e, 255), e)
            for t, out, unit in ((codes, self.codes, 16), (e, self.exps, 1)):
                if slots_first:
                    t = t.transpose(1, 2).contiguous().transpose(1, 2)
                if pad:      # blocks between a slot's and the next one's
                    wide = torch.zeros((*t.shape[:3], t.shape[3] + pad * unit), dtype=torch.uint8).cuda()
                    wide[..., :t.shape[3]] = t.cuda()
                    t = wide[..., :t.shape[3]]
                out.append(t.cuda())

    def cache(self):
        return pc.PagedCache(self.codes[0].view(FP4), self.codes[1].view(FP4), *self.exps)

    def run(self, causal=True, window=0, scale=None, **kw):
        kw.setdefault("max_q", int(self.new.max()) if len(self.new) else 0)
        kw.setdefault("want_lse", True)
        return pc.attn_paged(self.q, self.cache(), self.d_table, self.d_kv, self.d_off, causal=causal, window=window, scale=scale,
                             weight=self.weight, **kw)

    def want(self, causal=True, window=0, scale=None):
        k, v = (turn_plain.fp4_values(c, e) for c, e in zip(self.codes, self.exps))
        scale = self.q.shape[2] ** -0.5 if scale is None else float(np.float32(scale))
        want, tol = kv_plain.attention(self.q, k, v, self.table, self.kv, self.q_off, scale, causal, window, self.weight, self.dtype)
        # Values of 4 bits are often exactly zero, so that a result can be nothing but the terms of weights next to
        # zero.  The base-2 exponential gives 0 for results below 2^-126, the smallest normal number: of a
        # sum of exponentials that is at least 1 (the largest's), each of n weights is off by at most 2^-126 for
        # it, the result by n 2^-126 times the largest value.
        tol[0][...] += max(self.kv, default=0) * 2.0 ** -126 * np.nan_to_num(np.abs(v)).max()
        return want, tol


@pytest.mark.parametrize("lengths", sorted(set(LENGTHS) - {"empty_rows"}))
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_lengths_and_types(lengths, dtype):
    kv, new = LENGTHS[lengths]
    Case4(kv, new, dtype=dtype, seed=len(lengths), weights=True).check()


def test_rows_that_see_nothing():
    c = Case4(*LENGTHS["empty_rows"], seed=3, weights=True)
    got = c.run()
    torch.cuda.synchronize()
    assert pc.workspace_status(got[3]) == 2
    want, tol = c.want()
    for x, y, t in zip(got, want, tol):
        x = x.cpu().double().numpy()
        assert np.array_equal(np.isinf(x), np.isinf(y)) and np.all(np.abs(x - y)[~np.isinf(y)] <= t[~np.isinf(y)])


@pytest.mark.parametrize("heads,kvh", [(1, 1), (3, 3), (14, 2), (33, 1), (40, 1)])
@pytest.mark.parametrize("new", [1, 5, 40])
def test_head_groups(heads, kvh, new):
    Case4([new + 100, new, new + 3], [new, new, 1], heads=heads, kvh=kvh, seed=heads + new, weights=True).check()


@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_head_dims(dim, new, dtype):
    Case4([170, 50], [new, new], heads=6, kvh=2, dim=dim, dtype=dtype, seed=dim, weights=True).check()


@pytest.mark.parametrize("page", [1, 5, 16, 24, 64, 1000])
@pytest.mark.parametrize("new", [1, 37])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 33), (False, 70)])
def test_pages_and_masks(page, new, causal, window):
    Case4([300, 77, new], [new] * 3, page=page, seed=page + new, weights=True).check(causal=causal, window=window)


@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("slots_first,pad", [(True, 0), (False, 1), (True, 2), (False, 3)])
def test_strides(dim, new, slots_first, pad):
    """Scales then begin at any byte."""
    Case4([200, 41], [new, new], dim=dim, seed=dim + pad, slots_first=slots_first, pad=pad, weights=True).check()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-37, 20.0])
@pytest.mark.parametrize("new", [1, 40])
def test_factors(scale, new):
    Case4([100, 41, 3000], [new] * 3, weights=True, seed=new).check(scale=scale)


@pytest.mark.parametrize("kv,new,heads,kvh", [([9000, 200], [1, 1], 8, 2), ([8400], [300], 16, 2), ([8300, 700, 9], [160, 150, 9], 16, 1),
                                              ([2000] + [60] * 20, [120] + [7] * 20, 8, 2), ([700] * 90, [1] * 90, 4, 2)])
def test_cut_sequences(kv, new, heads, kvh):
    """Ranges of keys that are joined; tall tiles of rows; ragged chunks; more than 64 sequences."""
    Case4(kv, new, heads=heads, kvh=kvh, dim=128 if len(new) < 4 else 64, page=16, seed=len(kv), weights=len(kv) < 50).check()


def test_what_is_not_finite_stays_where_it_is_seen():
    """Blocks whose scale is NaN: in values and keys, in slots that all rows see, some see and none sees."""
    for new in (1, 6, 40):
        for place, which in ((10, 1), (199, 1), (120, 0), (196, 0)):
            c = Case4([200, 60], [new, new], dim=128, seed=place)
            page = c.table[0, place // c.page]
            c.exps[which][page, 1, place % c.page, 2] = 255
            c.check()
            if new > 1:
                c.check(window=30)


def test_scales_of_any_size():
    """The smallest and the largest exponent bytes; those that float16 has no numbers for."""
    c = Case4([90, 33], [1, 5], dtype=BF16, seed=1)
    for x in c.exps:
        x[x < 255] = 100 + (x[x < 255] % 3)
    c.exps[1][c.exps[1] < 255] -= 99             # values of 2^-126 and below: results are zero or next to it
    got = c.run()
    want, _ = c.want()
    assert np.all(np.abs(got[0].cpu().double().numpy() - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -124)
    assert np.array_equal(got[1].cpu().double().numpy().round(2), want[1].round(2))
    c = Case4([90, 33], [1, 5], dtype=F16, seed=1)
    c.exps[0][c.exps[0] < 255] = 103             # half of it is below float16's smallest number, times one it is that
    c.exps[1][c.exps[1] < 255] = 143             # times one it is above the largest
    got = c.run()
    v = turn_plain.fp4_values(c.codes[1], c.exps[1])
    assert np.isfinite(v[~np.isnan(v)]).all() and not np.isfinite(got[0].cpu().numpy()).all()


def test_results_in_place_and_between_queries():
    c = Case4([200, 90], [5, 5], heads=8, kvh=2, seed=9)
    want = c.run()[0].clone()
    assert torch.equal(c.run(out=c.q)[0], want)


def test_calls_repeat_exactly_on_two_streams():
    a, b = (Case4([3000, 500], [new, 1], heads=8, kvh=2, dim=128, seed=new, weights=True) for new in (1, 200))
    want = [[x.clone() for x in c.run()[:3]] for c in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for c, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                got.append(c.run()[:3])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_offsets_past_32_bits():
    """Codes past 4 GiB, scales past 2^28 bytes, in the last of many pages."""
    page, kvh, dim, pages = 1024, 4, 128, 17000
    codes = [torch.empty((pages, kvh, page, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = [torch.full((pages, kvh, page, dim // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert codes[0].numel() > 1 << 32
    g = torch.Generator().manual_seed(1)
    kv, ids = 1500, [pages - 1, pages - 2]
    k, v = (torch.randn((1500, kvh, dim), generator=g).to(BF16).cuda() for _ in range(2))
    cache = pc.PagedCache(codes[0].view(FP4), codes[1].view(FP4), *exps)
    ws = pc.kv_append(cache, i32([ids]), i32([kv]), i32([0, kv]), k, v)
    assert pc.workspace_status(ws) == 0
    q = torch.randn((1, 8, dim), generator=g).to(BF16).cuda()
    out, lse, _, ws = pc.attn_paged(q, cache, i32([ids]), i32([kv]), i32([0, 1]), 1, want_lse=True)
    assert pc.workspace_status(ws) == 0
    small = [turn_plain.fp4_values(c[ids], e[ids]) for c, e in zip(codes, exps)]
    want, tol = kv_plain.attention(q, *small, np.array([[0, 1]]), [kv], [0, 1], dim ** -0.5, True, 0)
    assert np.all(np.abs(out.cpu().double().numpy() - want[0]) <= tol[0])
    assert np.all(np.abs(lse.cpu().double().numpy() - want[1]) <= tol[1])
    assert bool((exps[0][:-2] == 255).all()) and bool((exps[1][ids[1], :, 1500 - 1024:] == 255).all())


@pytest.mark.parametrize("dim", [32, 96, 128])
@pytest.mark.parametrize("budget,recent", [(1, 1), (20, 5), (700, 0), (5000, 10)])
@pytest.mark.parametrize("slots_first", [False, True])
def test_evict(dim, budget, recent, slots_first):
    """Kept slots move with their codes and their scales, bit for bit."""
    g = torch.Generator().manual_seed(budget + recent)
    kv = np.array([0, 1, 64, 65, 1500, 4100])
    page, kvh = 24, 2
    table, pages = tables(kv, page, g)
    cols = (budget + page - 1) // page
    dst = torch.randperm(len(kv) * cols, generator=g).numpy().reshape(len(kv), cols) + pages
    both = []
    for width in (dim // 2, dim // 32):
        for _ in range(2):
            x = torch.randint(0, 256, (pages + dst.size, page, kvh, width), generator=g).to(torch.uint8)
            both.append(x.cuda().transpose(1, 2) if slots_first else x.transpose(1, 2).contiguous().cuda())
    w = weights("random", (len(kv), kvh, int(kv.max())), g)
    before = [x.cpu().numpy().copy() for x in both]
    got = pc.kv_evict(pc.PagedCache(both[0].view(FP4), both[1].view(FP4), *both[2:]), i32(table), i32(kv), w.cuda(), budget, recent,
                      dst_table=i32(dst))
    torch.cuda.synchronize()
    assert pc.workspace_status(got["ws"]) == 0
    kept, _, new_len = kv_plain.evict(w.numpy(), kv, budget, recent)
    assert np.array_equal(got["kept"].cpu().numpy(), kept)
    for x, b in zip(both, before):
        for s in range(len(kv)):
            for h in range(kvh):
                n = int(new_len[s])
                j, r = kept[s, h, :n], np.arange(n)
                b[dst[s, r // page], h, r % page] = b[table[s, j // page], h, j % page]
        assert np.array_equal(x.cpu().numpy(), b)


def test_a_session_as_it_is_used():
    """Prompts, decode steps that turn their tokens on the way and accumulate weights, an eviction, and more steps
    whose positions run ahead of their slots, over one cache in 4 bits: every step's attention is the definition's
    over what the cache then holds, and the cache holds the turned keys' nearest codes."""
    g = torch.Generator().manual_seed(11)
    heads, kvh, dim, page, n = 8, 2, 64, 16, 3
    codes = [torch.zeros((80, kvh, page, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = [torch.zeros((80, kvh, page, dim // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = pc.PagedCache(codes[0].view(FP4), codes[1].view(FP4), exps[0], exps[1])
    angles = pc.rope_table(pc.rope_frequencies(dim, scaling="ramp", factor=2.0, trained=128), 400)
    order = torch.randperm(80, generator=g).numpy()
    table, at = order[:60].reshape(n, 20).copy(), np.zeros(n, np.int64)
    text = np.zeros(n, np.int64)
    weight = torch.zeros((n, kvh, 320), device="cuda")

    def step(new):
        nonlocal weight
        new = np.array(new)
        off = np.concatenate([[0], np.cumsum(new)])
        pos = np.concatenate([np.arange(t, t + m) for t, m in zip(text, new)])
        fused = torch.randn((int(off[-1]), heads + 2 * kvh, dim), generator=g).to(BF16).cuda()
        q, k, v = fused.split([heads, kvh, kvh], 1)
        at[:] += new
        text[:] += new
        q, ws = pc.kv_append_rope(cache, i32(table), i32(at), i32(off), k, v, angles, pos=i32(pos), q=q, q_out=q)
        assert pc.workspace_status(ws) == 0
        before = weight
        out, lse, weight, ws = pc.attn_paged(q, cache, i32(table), i32(at), i32(off), int(new.max()), weight=before, want_lse=True)
        assert pc.workspace_status(ws) == 0
        ck, cv = (turn_plain.fp4_values(c, e) for c, e in zip(codes, exps))
        want, tol = kv_plain.attention(q, ck, cv, table, at, off, dim ** -0.5, True, 0, before)
        for x, y, t in zip((out, lse, weight), want, tol):
            assert np.all(np.abs(x.cpu().double().numpy() - y) <= t)
        turned, _ = turn_plain.turned(k.cpu().double(), angles, pos, False)
        held, _, _ = turn_plain.to_fp4(turned, BF16)
        for s in range(n):
            for i in range(new[s]):
                j = at[s] - new[s] + i
                assert np.array_equal(ck[table[s, j // page], :, j % page], held[off[s] + i])
    step([130, 1, 57])
    for _ in range(3):
        step([1, 1, 1])
    dst = order[60:80].reshape(1, 20)[:, :4]
    r = pc.kv_evict(cache, i32(table[:1]), i32(at[:1]), weight[:1].contiguous(), 60, 8, dst_table=i32(dst))
    assert pc.workspace_status(r["ws"]) == 0 and r["new_len"].tolist() == [60]
    table[0, :4], table[0, 4:20], at[0] = dst[0], order[64:80], 60
    weight[0] = 0
    weight[0, :, :60] = r["weight"][0]
    for new in ([1, 1, 1], [40, 0, 3], [1, 1, 0]):
        step(new)


def test_weights_of_more_scores_than_are_kept():
    """Few rows with room for more than 2^30 scores: the weights take a second pass over the keys."""
    n, kvh, page = 64, 8, 1000
    r = np.random.default_rng(5)
    kv = r.integers(1, 300, n)
    c = Case4(list(kv), [min(4, int(x)) for x in kv], heads=64, kvh=kvh, dim=32, page=page, seed=5, weights=True, cols=66)
    c.check()


def test_the_example_runs_over_4_bits():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_sessions.py")
    spec = importlib.util.spec_from_file_location("paged_sessions", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    server = example.run(sessions=4, steps=10, budget=96, recent=16, seed=2, cache="fp4")
    torch.cuda.synchronize()
    assert server.evictions >= 3 and server.len.max() <= 96 + 4 * 16 + 12 and bool((server.text > server.len).any())
    q, table, kv_len, q_off, out = server.last
    k, v = (turn_plain.fp4_values(x, e) for x, e in ((server.cache.k, server.cache.k_scale), (server.cache.v, server.cache.v_scale)))
    (want, _, _), (tol, _, _) = kv_plain.attention(q, k, v, table.cpu().numpy(), kv_len.cpu().numpy(), q_off.cpu().numpy(),
                                                   q.shape[2] ** -0.5, True, 0)
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= tol)


def test_binding_refuses():
    codes = torch.zeros((4, 2, 16, 32), dtype=torch.uint8, device="cuda")
    e = torch.zeros((4, 2, 16, 2), dtype=torch.uint8, device="cuda")
    k = codes.view(FP4)
    pc.PagedCache(k, codes.clone().view(FP4), e, e.clone())

    def refused(*args):
        with pytest.raises(pc.PcError):
            pc.PagedCache(*args)
    refused(k, k)
    refused(k, k, e)
    refused(codes, codes, e, e)
    refused(k, k, e.float(), e.float())
    refused(k, k, e[..., :1], e)
    refused(k, k, e, e.cpu())
    refused(k, k, e, e.transpose(1, 2).contiguous().transpose(1, 2))
    refused(k, k, torch.zeros((2,), device="cuda"), torch.zeros((2,), device="cuda"))
    odd = torch.zeros((4, 2, 16, 24), dtype=torch.uint8, device="cuda").view(FP4)      # head_dim 48
    refused(odd, odd, e[..., :1], e[..., :1])
    x = torch.zeros((4, 2, 16, 64), dtype=BF16, device="cuda")
    refused(x, x, e, e)
    cache = pc.PagedCache(k, codes.clone().view(FP4), e, e.clone().view(torch.float8_e8m0fnu))
    assert cache.head_dim == 64
    q = torch.zeros((1, 4, 64), dtype=BF16, device="cuda")
    ok = dict(page_table=i32([[0, 1]]), kv_len=i32([9]), q_off=i32([0, 1]), max_q=1)
    pc.attn_paged(q, cache, **ok)
    with pytest.raises(pc.PcError):
        pc.attn_paged(q[..., :32].contiguous(), cache, **ok)
    with pytest.raises(pc.PcError):
        pc.attn_paged(q.view(torch.uint8).view(torch.float8_e4m3fn)[..., :64], cache, **ok)
