"""Attention over a cache in 4 bits beside test_attn_fp4_gpu.py: items so long that a wave reads its table entries in
several goes, and what float16 holds of the smallest and the largest values.

Bounds as in kv_plain.py."""
import numpy as np
import pytest
import torch

import kv_plain
import turn_plain
from paper_2609_28870_amd import pc
from test_attn_fp4_gpu import BF16, F16, FP4, Case4
from test_kv_gpu import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def compare(got, want, tol):
    for name, x, y, t in zip(("out", "lse", "weight"), got, want, tol):
        x = x.cpu().double().numpy()
        fine = np.isfinite(y)
        assert np.array_equal(np.isnan(x), np.isnan(y)), name
        assert np.array_equal(x[~fine & ~np.isnan(y)], y[~fine & ~np.isnan(y)]), name
        over = np.abs(x[fine] - y[fine]) - t[fine]
        assert over.size == 0 or over.max() <= 0, (name, float(over.max()))


class Shared:
    """Many sequences whose tables draw on the same few pages: 1,024 pairs of a sequence and a head, which the
    list of items does not cut unless a sequence is much longer than the mean."""
    SEQS, KVH = 128, 8

    def __init__(self, lengths, group, dim, page, seed):
        g = torch.Generator().manual_seed(seed)
        r = np.random.default_rng(seed)
        pages = 16000 // page
        self.kv = np.resize(lengths, self.SEQS)
        cols = int((self.kv.max() + page - 1) // page)
        self.table = r.integers(0, pages, (self.SEQS, cols))
        self.bytes = [turn_plain.pack_fp4(torch.randn((pages, self.KVH, page, dim), generator=g).numpy(), BF16) for _ in range(2)]
        (k, ke), (v, ve) = ([x.cuda() for x in pair] for pair in self.bytes)
        self.cache = pc.PagedCache(k.view(FP4), v.view(FP4), ke, ve)
        self.q = torch.randn((self.SEQS, group * self.KVH, dim), generator=g).to(BF16).cuda()
        self.off, self.scale, self.page = np.arange(self.SEQS + 1), 6 * dim ** -0.5, page

    def run(self, window):
        out, lse, w, ws = pc.attn_paged(self.q, self.cache, i32(self.table), i32(self.kv), i32(self.off), 1, scale=self.scale,
                                        window=window, want_lse=True,
                                        weight=torch.zeros((self.SEQS, self.KVH, self.table.shape[1] * self.page), device="cuda"))
        assert pc.workspace_status(ws) == 0
        return out, lse, w

    def check(self, seqs, window=0):
        """Some of the sequences: scores are spread widely (the factor), so that a few keys make a row's result, and the
        weights name every key."""
        got = self.run(window)
        k, v = (turn_plain.fp4_values(*pair) for pair in self.bytes)
        want, tol = kv_plain.attention(self.q[seqs], k, v, self.table[seqs], self.kv[seqs], np.arange(len(seqs) + 1),
                                       float(np.float32(self.scale)), True, window, torch.zeros_like(got[2][seqs]))
        compare([x[seqs] for x in got], want, tol)


@pytest.mark.parametrize("dim,group,page", [(64, 1, 16), (64, 20, 48), (128, 3, 16), (128, 17, 64), (192, 2, 16), (256, 1, 1024)])
def test_items_of_many_tiles(dim, group, page):
    """A wave keeps the entries of 32 tiles (of a workgroup 4,096 keys) and reads on: once, twice, and in ranges of a
    sequence that is cut."""
    c = Shared([4200, 8900, 4097, 4096, 12300, 6000, 5], group, dim, page, seed=dim + group)
    c.check([0, 1, 2, 3, 4, 6, 127])
    c.check([1, 4], window=8500)
    c.kv[9] = 30000
    c.table = np.random.default_rng(1).integers(0, 16000 // page, (c.SEQS, 30000 // page + 1))
    c.check([8, 9, 126])


def float16_of(codes, exponents):
    with np.errstate(over="ignore"):
        return turn_plain.fp4_values(codes, exponents).astype(np.float16).astype(np.float64)


@pytest.mark.parametrize("new", [[1, 5], [40, 33]], ids=["few", "chunk"])
def test_float16_of_the_smallest_keys(new):
    """Scales of 2^-24: half of it is a tie that goes to 0, one and a half times it one that goes to 2^-23; and of
    2^-22, where nothing is rounded."""
    for exponent in (103, 105):
        c = Case4([90, 53], new, dtype=F16, seed=exponent, weights=True)
        c.exps[0][c.exps[0] < 255] = exponent
        got = c.run(scale=2.0 ** 20)
        k, v = float16_of(c.codes[0], c.exps[0]), float16_of(c.codes[1], c.exps[1])
        want, tol = kv_plain.attention(c.q, k, v, c.table, c.kv, c.q_off, 2.0 ** 20, True, 0, c.weight, F16)
        compare(got, want, tol)


@pytest.mark.parametrize("new", [[1, 5], [40, 33]], ids=["few", "chunk"])
def test_float16_of_the_largest_values(new):
    """Scales of 2^16: half of it is a number, once it is above the largest, so infinite, for the rows that see it
    and in its dimension alone."""
    c = Case4([90, 53], new, dtype=F16, seed=4)
    e = c.exps[1]
    e[e < 255] = 143
    low = torch.randint(0, 4, (*c.codes[1].shape[:3], 32), generator=torch.Generator().manual_seed(5), dtype=torch.uint8)
    low = torch.where(low < 2, low, low + 6)                                # 0, 0.5, and their negatives
    high = torch.randint(0, 40, (*low.shape[:3], 32), generator=torch.Generator().manual_seed(6), dtype=torch.uint8)
    high = torch.where(high > 7, torch.zeros_like(high), high)             # some of 0.5 to 6
    both = torch.cat([low, high], 3)
    c.codes[1] = (both[..., ::2] | both[..., 1::2] << 4).cuda()
    got = c.run()
    k, v = float16_of(c.codes[0], c.exps[0]), float16_of(c.codes[1], e)
    want, tol = kv_plain.attention(c.q, k, v, c.table, c.kv, c.q_off, 64 ** -0.5, True, 0, None, F16)
    assert np.isinf(want[0][..., 32:]).any() and np.isfinite(want[0][..., :32]).all()
    # subnormal weights: kv_plain counts them against the largest value, which is infinite here; finite ones are 2^15
    tol[0][...] = 2.0 ** -11 * np.abs(np.nan_to_num(want[0], posinf=0.0)) + (2.0 ** -11 + 2.0 ** -15) * 2.0 ** 15
    compare(got[:2], want[:2], tol[:2])


@pytest.mark.parametrize("new", [1, 40])
def test_results_between_queries(new):
    c = Case4([200, 90], [new, new], heads=8, kvh=2, seed=9)
    want = c.run()[0].clone()
    wide = torch.full((2 * new, 8, 2, 64), 3.0, dtype=BF16, device="cuda")
    wide[:, :, 0] = c.q
    before, c.q = c.q.clone(), wide[:, :, 0]
    out = c.run(out=wide[:, :, 1])[0]
    assert torch.equal(out, want) and torch.equal(wide[:, :, 0], before) and torch.equal(wide[:, :, 1], want)
