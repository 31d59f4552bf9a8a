"""pc_rope_table, pc_rope and pc_kv_append_rope against their definitions in 64 bits: layouts, parts
of heads, types, positions, strides, streams, graphs, refusals.

Bounds.  The angles that a table is compared with are products in 80 bits, off by 2^-64 of themselves; the library's are
exact, their reduction, the series and the turns from one position to the next off by less than 1e-13 together, the
rounding to 32 bits by 2^-24 of the result.  A turned element is a sum of two
products in 32 bits (one rounding of a product, one of the sum: 2^-24 of the sum of their magnitudes each),
rounded to the type: half a step, u = 2^-9 or 2^-12 of it (2^-25 of a float16 below its normal range);
twice that is allowed, for a sum that lies next to a border.  Codes of 8 and 4 bits are taken of the exact
sum rounded to 32 bits: they are equal.
"""
import numpy as np
import pytest
import torch

import kv_plain
import turn_plain
from paper_2609_28870_amd import pc
from test_kv_gpu import bits, i32, tables

pytestmark = pytest.mark.gpu
BF16, F16, FP8, FP4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.float4_e2m1fn_x2
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def rows(shape, dtype, g, size=2.0):
    return (torch.randn(shape, generator=g) * size).to(dtype).cuda()


def near(got, want, size, dtype):
    got = got.cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    tol = (U[dtype] * np.abs(want) + 2.0 ** -23 * size + (2.0 ** -24 if dtype == F16 else 0))[fine]
    off = np.abs(got[fine] - want[fine])
    assert np.all(off <= tol), float(np.max(off - tol))


# -------------------------------------------------------------------- table

@pytest.mark.parametrize("pairs", [1, 3, 16, 64, 100, 128])
@pytest.mark.parametrize("n_pos,first", [(1, 0), (2, 1), (1000, 0), (777, 131072), (65, (1 << 31) - 3), (3, 0xFFFFFFF0)])
def test_table(pairs, n_pos, first):
    freq = pc.rope_frequencies(2 * pairs, 10000.0, "ramp", 8.0, trained=4096)
    freq[0] = -1.5 if pairs > 1 else 1.0
    got = pc.rope_table(freq, n_pos, first=first, magnitude=1.1).cpu().numpy().astype(np.float64)
    a = np.multiply.outer(first + np.arange(n_pos, dtype=np.longdouble), freq.astype(np.longdouble))    # 64 bits of fraction
    want = (1.1 * np.stack([np.cos(a), np.sin(a)], -1)).astype(np.float64)
    assert got.shape == (n_pos, pairs, 2)
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2e-13 + 2.0 ** -63 * np.abs(a.astype(np.float64))[..., None])


def test_table_of_nothing_and_refusals():
    assert pc.rope_table(np.ones(4), 0).shape == (0, 4, 2)
    out = torch.zeros((5, 4, 2), device="cuda")
    assert pc.rope_table(np.zeros(4), 5, out=out) is out and bool((out[..., 0] == 1).all()) and bool((out[..., 1] == 0).all())
    for kw in (dict(freq=np.ones((2, 2))), dict(n_pos=-1), dict(first=-1), dict(first=1 << 32), dict(out=out[:4]),
               dict(out=out.double()), dict(magnitude=float("nan")), dict(freq=np.full(4, np.nan)), dict(freq=np.ones(129)),
               dict(n_pos=1 << 33)):
        with pytest.raises(pc.PcError):
            pc.rope_table(**dict(dict(freq=np.ones(4), n_pos=5), **kw))


# --------------------------------------------------------------------- rope

@pytest.mark.parametrize("dim,rot", [(8, 2), (8, 8), (16, 6), (64, 64), (64, 16), (80, 20), (80, 80), (96, 24), (96, 64), (128, 128),
                                     (128, 32), (256, 256), (256, 66)])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_rows(dim, rot, interleaved, dtype):
    g = torch.Generator().manual_seed(dim + rot)
    table = turn_plain.angles(500, rot, magnitude=1.2 if rot == 64 else 1.0)
    for n, heads in ((1, 1), (37, 3), (300, 9)):
        x, pos = rows((n, heads, dim), dtype, g), torch.randint(0, 500, (n,), generator=g)
        for transpose in (False, True):
            got, ws = pc.rope(x, table, i32(pos), interleaved=interleaved, transpose=transpose)
            assert pc.workspace_status(ws) == 0
            want, size = turn_plain.turned(x.cpu().double(), table, pos, interleaved, transpose)
            near(got, want, size, dtype)
        own = pc.rope(x, table, interleaved=interleaved)[0]          # row t at position t
        assert torch.equal(own, pc.rope(x, table, i32(np.arange(n)), interleaved=interleaved)[0])
        again = x.clone()
        assert pc.rope(again, table, interleaved=interleaved, out=again)[0] is again and torch.equal(again, own)


@pytest.mark.parametrize("n", [32768, 32769, 70001])
@pytest.mark.parametrize("heads,dim,rot,interleaved", [(1, 16, 16, False), (5, 8, 4, True), (2, 24, 10, False)])
def test_many_rows(n, heads, dim, rot, interleaved):
    """On either side of the number of rows whose positions one workgroup looks at."""
    g = torch.Generator().manual_seed(n)
    table = turn_plain.angles(300, rot)
    x, pos = rows((n, heads, dim), BF16, g), torch.randint(0, 300, (n,), generator=g)
    got, ws = pc.rope(x, table, i32(pos), interleaved=interleaved)
    assert pc.workspace_status(ws) == 0
    near(got, *turn_plain.turned(x.cpu().double(), table, pos, interleaved), BF16)
    for at in (0, n // 2, n - 1):
        past = i32(pos)
        past[at] = 300
        out = torch.full_like(x, 7.0)
        got2, ws = pc.rope(x, table, past, interleaved=interleaved, out=out)
        assert pc.workspace_status(ws) == 2
        want = got.clone()
        want[at] = 7.0
        assert torch.equal(got2, want)
    assert pc.workspace_status(pc.rope(x, table, i32(pos), interleaved=interleaved, ws=ws)[1]) == 0


def test_many_heads_and_strides():
    """Threads that take several heads; rows of a fused projection, heads before rows, results between them."""
    g = torch.Generator().manual_seed(5)
    for heads, dim, rot, interleaved in ((40, 128, 128, False), (33, 64, 32, True), (7, 96, 24, False), (130, 32, 32, True)):
        table = turn_plain.angles(900, rot)
        n = 2500 if heads < 100 else 700
        fused = rows((n, heads + 5, dim), BF16, g)
        x, pos = fused[:, 2:2 + heads], torch.randint(0, 900, (n,), generator=g)
        want, size = turn_plain.turned(x.cpu().double(), table, pos, interleaved)
        got = pc.rope(x, table, i32(pos), interleaved=interleaved)[0]
        near(got, want, size, BF16)
        first = x.transpose(0, 1).contiguous().transpose(0, 1)               # [head, row, dim]
        out = torch.empty_like(first)
        assert torch.equal(pc.rope(first, table, i32(pos), interleaved=interleaved, out=out)[0], got)
        before = fused.clone()
        pc.rope(x, table, i32(pos), interleaved=interleaved, out=x)          # in place: the rest of the rows stays
        before[:, 2:2 + heads] = got
        assert torch.equal(fused, before)


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("rot", [64, 24])
def test_gradient(interleaved, rot):
    """Transposed, it is the gradient: against autograd of the formula, and against differences."""
    g = torch.Generator().manual_seed(rot)
    table, pos = turn_plain.angles(100, rot, magnitude=1.3), torch.randint(0, 100, (50,), generator=g)
    x, dy = rows((50, 4, 64), BF16, g), rows((50, 4, 64), BF16, g)
    a, b = (torch.from_numpy(d) for d in turn_plain.pair_of(rot, interleaved))
    z = x.cpu().double().requires_grad_()
    c, s = table.cpu().double()[pos][:, None].unbind(-1)
    y = z.clone()
    y[..., a] = z[..., a] * c - z[..., b] * s
    y[..., b] = z[..., b] * c + z[..., a] * s
    (y * dy.cpu().double()).sum().backward()
    got = pc.rope(dy, table, i32(pos), interleaved=interleaved, transpose=True)[0]
    _, size = turn_plain.turned(dy.cpu().double(), table, pos, interleaved, True)
    near(got, z.grad.numpy(), size, BF16)
    # the map is linear: a difference over any step is its derivative, up to the roundings of the two results
    h = rows((50, 4, 64), BF16, g)
    far = (x.float() + h.float()).to(BF16)
    step = far.double() - x.double()
    up, low = (pc.rope(v, table, i32(pos), interleaved=interleaved)[0].double() for v in (far, x))
    lhs, rhs = ((up - low) * dy.double()).sum(), (got.double() * step).sum()
    tol = 2.0 ** -8 * (((up.abs() + low.abs()) * dy.double().abs()).sum() + (got.double().abs() * step.abs()).sum())
    assert abs(float(lhs - rhs)) <= float(tol)


def test_what_is_not_finite():
    """It stays in its pair, and out of the part that does not turn."""
    table, dim, rot = turn_plain.angles(50, 16), 32, 16
    for interleaved in (False, True):
        x = torch.randn((50, 2, dim), generator=torch.Generator().manual_seed(1)).to(F16)
        x[3, 0, 5], x[4, 1, 12], x[5, 0, 30], x[6, 1, 0] = float("nan"), float("inf"), float("nan"), float("-inf")
        x = x.cuda()
        want, size = turn_plain.turned(x.cpu().double(), table, np.arange(50), interleaved)
        near(pc.rope(x, table, interleaved=interleaved)[0], want, np.nan_to_num(size), F16)


def test_rope_of_nothing_and_refusals():
    table = turn_plain.angles(20, 8)
    x = torch.ones((6, 2, 16), dtype=BF16, device="cuda")
    out, ws = pc.rope(x[:0], table, i32([]))
    assert out.shape == (0, 2, 16) and pc.workspace_status(ws) == 0
    ok = dict(x=x, table=table, pos=i32([0] * 6))
    pc.rope(**ok)

    def refused(**kw):
        with pytest.raises(pc.PcError):
            pc.rope(**dict(ok, **kw))
    refused(x=x.float())
    refused(x=x.to(FP8))
    refused(x=x[0])
    refused(x=torch.ones((6, 2, 12), dtype=BF16, device="cuda"))
    refused(x=torch.ones((6, 16, 2), dtype=BF16, device="cuda").transpose(1, 2))
    refused(x=x.cpu())
    refused(x=x.clone().requires_grad_())
    refused(x=torch.ones((6, 2, 20), dtype=BF16, device="cuda")[..., 4:])
    refused(table=table.double())
    refused(table=table[..., 0])
    refused(table=table.cpu())
    refused(table=turn_plain.angles(20, 18))                    # more dimensions than a head has
    refused(table=table[:0])
    refused(pos=None, table=table[:5])
    refused(pos=i32([0] * 5))
    refused(pos=torch.zeros(6, dtype=torch.int64, device="cuda"))
    refused(out=x.to(F16))
    refused(out=x[:5])
    refused(ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    fused = torch.ones((7, 2, 16), dtype=BF16, device="cuda")
    refused(x=fused[:6], out=fused[1:])
    with torch.no_grad():
        pc.rope(x.clone().requires_grad_(), table)


# ------------------------------------------------------------------- append

class Append:
    """Pages, new rows and positions of one call, and what it has to leave behind."""

    def __init__(self, kv, new, page=16, dtype=BF16, cache=None, heads=4, kvh=2, dim=64, rot=None, interleaved=False, given=False,
                 seed=0, slots_first=False, size=2.0):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.new, self.dtype, self.cache = np.array(kv), np.array(new), dtype, cache or dtype
        self.interleaved, self.page = interleaved, page
        self.off = np.concatenate([[0], np.cumsum(new)])
        self.table, pages = tables(self.kv, page, g)
        n, rot = int(self.off[-1]), rot or dim
        self.n_pos = int(self.kv.max()) + 40 if len(kv) else 40
        self.angles = turn_plain.angles(self.n_pos, rot)
        slots = np.concatenate([np.arange(c - m, c) for c, m in zip(self.kv, self.new)] + [[]]).astype(np.int64)
        self.pos = torch.randint(0, self.n_pos, (n,), generator=g).numpy() if given else slots
        self.given = given
        fused = rows((n, heads + 2 * kvh, dim), dtype, g, size)
        self.fused = fused
        self.q, self.k, self.v = fused.split([heads, kvh, kvh], 1)
        width = dim // 2 if self.cache == FP4 else dim
        x = torch.randint(0, 256, (2, pages, kvh, page, width), generator=g)
        self.scales = [None, None]
        if self.cache == FP4:
            e = torch.randint(0, 256, (2, pages, kvh, page, dim // 32), generator=g).to(torch.uint8)
            if slots_first:
                e = e.transpose(2, 3).contiguous().cuda().transpose(2, 3)
            self.scales = [e[0].cuda(), e[1].cuda()]
        elif self.cache == FP8:
            self.scales = [(0.01 + torch.rand(kvh, generator=g)).cuda() for _ in range(2)]
        if self.cache in (FP4, FP8):
            x = x.to(torch.uint8).view(self.cache)
        else:
            x = torch.randn(x.shape, generator=g).to(self.cache)
        if slots_first:
            x = x.view(torch.uint8 if self.cache in (FP4, FP8) else self.cache).transpose(2, 3).contiguous().cuda().transpose(2, 3)
            x = x.view(self.cache) if self.cache in (FP4, FP8) else x
        self.pages = [x[0].cuda(), x[1].cuda()]

    def run(self, **kw):
        kw.setdefault("q", self.q)
        kw.setdefault("pos", i32(self.pos) if self.given else None)
        return pc.kv_append_rope(pc.PagedCache(*self.pages, *self.scales), i32(self.table), i32(self.kv), i32(self.off), self.k, self.v,
                                 self.angles, interleaved=self.interleaved, **kw)

    def stored(self):
        """Bits of both caches (and of their scales)."""
        return [bits(x.view(torch.uint8) if x.dtype == FP4 else x).cpu().numpy().copy() for x in self.pages + [
            s for s in self.scales if s is not None and self.cache == FP4]]

    def want(self, lost=()):
        out = self.stored()
        k, _ = turn_plain.turned(self.k.cpu().double(), self.angles, np.minimum(self.pos, self.n_pos - 1), self.interleaved)
        k16 = pc.rope(self.k, self.angles, i32(np.minimum(self.pos, self.n_pos - 1)), interleaved=self.interleaved)[0]
        for i, (exact, rows16) in enumerate(((k, k16), (self.v.cpu().double().numpy(), self.v))):
            if self.cache == FP4:
                codes, e = turn_plain.pack_fp4(exact, self.dtype)
                codes = codes.numpy()
                put = [(out[i], codes), (out[2 + i], e.numpy())]
            elif self.cache == FP8:
                y = exact.astype(np.float32) / self.scales[i].cpu().numpy()[None, :, None]
                put = [(out[i], torch.from_numpy(kv_plain.nearest_e4m3(y.astype(np.float64))).float().to(FP8).view(torch.uint8).numpy())]
            else:
                put = [(out[i], bits(rows16.contiguous()).cpu().numpy())]
            for s in range(len(self.kv)):
                for r in range(self.new[s]):
                    t, j = self.off[s] + r, self.kv[s] - self.new[s] + r
                    if t in lost or j < 0:
                        continue
                    for x, y in put:
                        x[self.table[s, j // self.page], :, j % self.page] = y[t]
        return out

    def check(self, **kw):
        want = self.want()
        q_out, ws = self.run(**kw)
        torch.cuda.synchronize()
        assert pc.workspace_status(ws) == 0
        got = self.stored()
        if self.cache == FP4:
            # the sign of a zero is open
            for x, y in ((0, got), (1, got), (0, want), (1, want)):
                c = y[x]
                c = np.where((c & 0x0F) == 0x08, c & 0xF0, c)
                y[x] = np.where((c & 0xF0) == 0x80, c & 0x0F, c)
        for x, y in zip(got, want):
            assert np.array_equal(x, y)
        if kw.get("q", self.q) is not None:
            assert torch.equal(q_out, pc.rope(self.q, self.angles, i32(self.pos), interleaved=self.interleaved)[0])
        return self


TYPES = [(BF16, BF16), (F16, F16), (BF16, FP8), (F16, FP8), (BF16, FP4), (F16, FP4)]
TYPE_IDS = ["bf16", "f16", "bf16-fp8", "f16-fp8", "bf16-fp4", "f16-fp4"]


@pytest.mark.parametrize("kv,new", [([1], [1]), ([17, 0, 40, 33], [1, 0, 1, 1]), ([50, 300, 24, 7], [50, 111, 1, 0]),
                                    (list(range(1, 140)), [1 + i % 3 if i > 3 else 1 for i in range(139)])],
                         ids=["one", "decode", "chunks", "many"])
@pytest.mark.parametrize("page", [1, 16, 24])
@pytest.mark.parametrize("dtype,cache", TYPES, ids=TYPE_IDS)
def test_append(kv, new, page, dtype, cache):
    Append(kv, new, page, dtype, cache, seed=len(kv) + page, slots_first=page == 24, given=page == 16).check()


@pytest.mark.parametrize("dim,rot", [(32, 32), (32, 6), (64, 16), (96, 24), (96, 96), (128, 128), (128, 64), (256, 256), (256, 130)])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("dtype,cache", TYPES, ids=TYPE_IDS)
def test_append_layouts(dim, rot, interleaved, dtype, cache):
    Append([70, 3, 0, 41], [33, 3, 0, 1], 10, dtype, cache, heads=6, kvh=3, dim=dim, rot=rot, interleaved=interleaved,
           given=rot % 32 == 0, seed=dim + rot).check()


@pytest.mark.parametrize("heads,kvh", [(1, 1), (40, 1), (12, 12), (130, 65)])
@pytest.mark.parametrize("cache", [BF16, FP8, FP4], ids=["bf16", "fp8", "fp4"])
def test_append_heads(heads, kvh, cache):
    Append([33, 20], [30, 1], 16, BF16, cache, heads=heads, kvh=kvh, seed=heads).check()


@pytest.mark.parametrize("cache", [BF16, FP4], ids=["bf16", "fp4"])
def test_queries_in_place_none_or_apart(cache):
    for change in ("in place", "none", "apart"):
        a = Append([60, 9], [20, 3], 16, BF16, cache, seed=7, given=True)
        want = pc.rope(a.q, a.angles, i32(a.pos))[0]
        if change == "in place":
            before = a.fused.clone()
            expect = a.want()
            out, ws = a.run(q_out=a.q)
            assert pc.workspace_status(ws) == 0 and torch.equal(a.q, want) and torch.equal(a.fused[:, 4:], before[:, 4:])
            assert torch.equal(torch.from_numpy(a.stored()[0]), torch.from_numpy(expect[0])) or cache == FP4
        elif change == "none":
            assert a.check(q=None).run(q=None)[0] is None
        else:
            out = torch.zeros((23, 9, 64), dtype=BF16, device="cuda")[:, 2:6]
            a.run(q_out=out)
            assert torch.equal(out, want)


@pytest.mark.parametrize("n_seqs", [1, 3, 70, 5000])
@pytest.mark.parametrize("cache,kvh,dim", [(BF16, 3, 80), (FP8, 4, 128), (FP4, 1, 32), (FP4, 4, 128)])
def test_append_many_rows(n_seqs, cache, kvh, dim):
    """Sequences of any length, many of them empty, more than 64 of them behind one another."""
    r = np.random.default_rng(n_seqs + dim)
    cut = np.sort(r.integers(0, 9002, n_seqs - 1))
    if n_seqs == 5000:
        cut[1000:1300] = cut[1000]                    # 300 empty ones in a row
    new = np.diff(np.concatenate([[0], np.sort(cut), [9001]]))
    Append(new + r.integers(0, 30, n_seqs), new, 24, BF16, cache, heads=kvh, kvh=kvh, dim=dim, seed=n_seqs).check()


def test_append_above_what_one_workgroup_looks_at():
    a = Append([33000, 5, 900], [32990, 1, 800], 64, F16, FP4, heads=1, kvh=1, dim=32, given=True, seed=3)
    a.check()
    a.pos[32990] = a.n_pos                             # the row of the second sequence
    q_out = torch.full_like(a.q.contiguous(), 5.0)
    want = a.want(lost={32990})
    _, ws = a.run(q_out=q_out)
    assert pc.workspace_status(ws) == 2 and bool((q_out[32990] == 5).all()) and not bool((q_out[32989] == 5).any())
    assert all(np.array_equal(x, y) for x, y in zip(a.stored()[2:], want[2:]))


@pytest.mark.parametrize("cache", [BF16, FP8, FP4], ids=["bf16", "fp8", "fp4"])
def test_append_leaves_out_what_does_not_fit(cache):
    def run(change, lost, given=False):
        a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2, given=given)
        a.q_out = torch.full_like(a.q.contiguous(), 9.0)
        right = a.run()[0].clone()
        a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2, given=given)
        change(a)
        want, n = a.want(lost=lost), 10
        q_out = torch.full_like(a.q.contiguous(), 9.0)
        _, ws = a.run(q_out=q_out)
        torch.cuda.synchronize()
        got = a.stored()
        if cache == FP4:
            got, want = got[2:], want[2:]
        assert all(np.array_equal(x, y) for x, y in zip(got, want))
        untouched = {t for t in range(n) if bool((q_out[t] == 9).all())}
        for t in set(range(n)) - untouched:
            assert torch.equal(q_out[t], right[t])
        return pc.workspace_status(ws), untouched

    def no_slot(a):
        a.kv[2] = 3

    def no_page(a):
        a.table[1] = 1 << 20

    def short_table(a):
        a.angles, a.n_pos = a.angles[:39], 39

    def far(a):
        a.pos[[2, 7]] = [a.n_pos, 0xFFFFFFFF - (1 << 32)]
    assert run(lambda a: None, ()) == (0, set())
    code, untouched = run(no_page, {3, 4})
    assert code == 2 and untouched == set()
    assert run(short_table, {2}) == (2, {2})
    # positions below 0 are large ones
    a_far = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2, given=True)
    far(a_far)
    q_out = torch.full_like(a_far.q.contiguous(), 9.0)
    assert pc.workspace_status(a_far.run(q_out=q_out)[1]) == 2
    assert {t for t in range(10) if bool((q_out[t] == 9).all())} == {2, 7}
    # rows before the first slot: the others' slots, and positions, shift with the length
    a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2)
    no_slot(a)
    q_out = torch.full_like(a.q.contiguous(), 9.0)
    assert pc.workspace_status(a.run(q_out=q_out)[1]) == 2
    assert {t for t in range(10) if bool((q_out[t] == 9).all())} == {5, 6}
    for off in ([0, 3, 2, 10], [0, 3, 5, 11], [2, 3, 5, 10]):
        a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2)
        a.off = np.array(off)
        assert pc.workspace_status(a.run()[1]) == 2
    a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2)
    assert pc.workspace_status(a.run(max_kv=39)[1]) == 2


def test_append_nothing():
    a = Append([2, 0], [0, 0], 16, BF16, FP4, seed=1)
    before = a.stored()
    q_out, ws = a.run()
    assert q_out.shape == (0, 4, 64) and pc.workspace_status(ws) == 0
    assert all(np.array_equal(x, y) for x, y in zip(a.stored(), before))
    none = a.k[:0]
    cache = pc.PagedCache(*a.pages, *a.scales)
    _, ws = pc.kv_append_rope(cache, i32(a.table[:0]), i32([]), i32([0]), none, none, a.angles)      # no sequences
    assert pc.workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_4_bit_codes_of_every_pattern(dtype):
    """Every 16-bit pattern beside its neighbours, beside larger ones, and every tie: subnormals, the largest
    numbers, infinities, NaN.  The plain append writes them, with no rotation."""
    dim, page = 64, 64
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).view(1024, 1, dim)
    small = torch.randn((512, 1, dim), generator=torch.Generator().manual_seed(3)).to(dtype)
    tie = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 6.98, 7.0, 0.0, -0.25, -0.75, -5.0, -3.5])
    ties = torch.stack([torch.cat([tie, tie]) * 2.0 ** (p % 24 - 10) for p in range(128)]).view(64, 1, dim).to(dtype)
    x = torch.cat([x, small, ties]).cuda()
    n = x.shape[0]
    table, pages = tables([n], page, torch.Generator().manual_seed(0))
    codes = torch.zeros((2, pages, 1, page, dim // 2), dtype=torch.uint8, device="cuda")
    e = torch.zeros((2, pages, 1, page, dim // 32), dtype=torch.uint8, device="cuda")
    cache = pc.PagedCache(codes[0].view(FP4), codes[1].view(FP4), e[0], e[1].view(torch.float8_e8m0fnu))
    ws = pc.kv_append(cache, i32(table), i32([n]), i32([0, n]), x, x)
    torch.cuda.synchronize()
    assert pc.workspace_status(ws) == 0
    want, _, exponents = turn_plain.to_fp4(torch.nan_to_num(x, nan=float("nan"), posinf=3.3e38 if dtype == BF16 else 65504,
                                                            neginf=-3.3e38 if dtype == BF16 else -65504).cpu().double().numpy(), dtype)
    at = i32(table)[0].long()
    for i in range(2):
        got = turn_plain.fp4_values(codes[i][at], e[i][at]).transpose(0, 2, 1, 3).reshape(-1, 1, dim)[:n]
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want))
        assert np.array_equal(e[i][at].cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, 2)[:n], exponents[:, 0])
        assert np.nanmax(np.abs(got)) <= torch.finfo(dtype).max


@pytest.mark.parametrize("cache", [BF16, FP4], ids=["bf16", "fp4"])
def test_step_replays_in_a_graph_and_on_a_stream(cache):
    """Append with rotation, then attention, captured once and replayed over other tokens and lengths."""
    kv, new = [200, 90, 0], [3, 1, 0]
    a = Append(kv, new, 16, BF16, cache, seed=4)
    table, n_kv, off = i32(a.table), i32(kv), i32(a.off)
    ws = [pc.workspace(256), pc.workspace(pc.lib().pc_attn_paged_ws(3, 4, 3, 208, 4, 2, 64, 0))]
    q_out, out = torch.empty_like(a.q.contiguous()), torch.empty_like(a.q.contiguous())
    paged = pc.PagedCache(*a.pages, *a.scales)

    def step():
        pc.kv_append_rope(paged, table, n_kv, off, a.k, a.v, a.angles, q=a.q, q_out=q_out, ws=ws[0])
        pc.attn_paged(q_out, paged, table, n_kv, off, 3, max_kv=208, out=out, ws=ws[1])
    # old tokens: whatever the pages hold, if it is finite
    base = []
    for x, s in zip(a.pages, a.scales):
        if cache == FP4:
            s.copy_(torch.randint(120, 130, s.shape, dtype=torch.uint8))
        else:
            x.copy_(torch.randn(x.shape).to(BF16))
    base = [x.view(torch.uint8).clone() if x.dtype == FP4 else x.clone() for x in a.pages + [s for s in a.scales if s is not None]]

    def restore():
        for x, y in zip(a.pages + [s for s in a.scales if s is not None], base):
            (x.view(torch.uint8) if x.dtype == FP4 else x).copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(9)
    for i in range(4):
        a.fused.copy_(torch.randn(a.fused.shape, generator=g).to(BF16))
        n_kv.copy_(i32([200 - 7 * i, 90 + i, 5 * i]))
        restore()
        step()
        want = [q_out.clone(), out.clone()] + a.stored()
        restore()
        q_out.zero_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [q_out, out] + a.stored()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert all(np.array_equal(x, y) for x, y in zip(got[2:], want[2:]))
        assert pc.workspace_status(ws[0]) == 0 and pc.workspace_status(ws[1]) == 0
        if i == 2:
            with torch.cuda.stream(side):
                side.wait_stream(torch.cuda.current_stream())
                restore()
                step()
            torch.cuda.synchronize()
            assert torch.equal(out, want[1])


def test_append_refusals():
    a = Append([9], [3], 16, BF16, BF16, seed=1)
    a.run()

    def refused(**kw):
        with pytest.raises(pc.PcError):
            a.run(**kw)
    refused(q=a.q.to(F16))
    refused(q=a.q[:2])
    refused(q=a.q[..., :32])
    refused(q=a.q[0])
    refused(q=a.q.clone().requires_grad_())
    refused(q_out=a.k)
    refused(q_out=a.fused[:, 1:5])
    refused(q_out=a.q.float())
    refused(q=None, q_out=a.q)
    refused(pos=i32([0, 1]))
    refused(pos=torch.zeros(3, dtype=torch.int64, device="cuda"))
    refused(max_kv=33)
    refused(ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    for name, bad in (("k", a.k.to(F16)), ("v", a.v[:2]), ("angles", turn_plain.angles(60, 66)), ("angles", a.angles.double()),
                      ("k", a.k.clone().requires_grad_())):
        good = getattr(a, name)
        setattr(a, name, bad)
        refused()
        setattr(a, name, good)
    with torch.no_grad():
        a.run(q=a.q.clone().requires_grad_())
