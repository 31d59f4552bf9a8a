"""Calls of the rotation and of caches in 4 bits beside those of test_rope_gpu.py and test_attn_fp4_gpu.py: other
layouts of a projection, every code and scale of a 4-bit cache compared, offsets past 32 bits."""
import pytest
import torch

import turn_plain
from paper_2609_28870_amd import pc
from test_kv_gpu import i32
from test_rope_gpu import BF16, F16, FP4, FP8, Append, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def plus_zero(codes):
    """Two codes a byte, the sign of a zero (which is open) taken away."""
    codes = torch.from_numpy(codes)
    codes = torch.where((codes & 0x0F) == 0x08, codes & 0xF0, codes)
    return torch.where((codes & 0xF0) == 0x80, codes & 0x0F, codes)


def same(a, got, want):
    """Everything that both caches hold: codes, and of a 4-bit cache scales."""
    assert len(got) == len(want) == (4 if a.cache == FP4 else 2)
    for i, (x, y) in enumerate(zip(got, want)):
        x, y = (plus_zero(z) if a.cache == FP4 and i < 2 else torch.from_numpy(z) for z in (x, y))
        assert torch.equal(x, y)


@pytest.mark.parametrize("cache", [BF16, FP8, FP4], ids=["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("new", [[1, 0, 0], [20, 3, 1], [700, 41, 1]])
def test_a_heads_query_key_and_value_beside_each_other(cache, new):
    """A projection of [row, head, 3, head_dim], its queries turned in place."""
    a = Append([new[0] + 5, 44, 9], new, 16, BF16, cache, heads=4, kvh=4, seed=sum(new), given=True)
    a.fused = rows((sum(new), 4, 3, 64), BF16, torch.Generator().manual_seed(8))
    a.q, a.k, a.v = a.fused.unbind(2)
    want, before = a.want(), a.fused.clone()
    turned = pc.rope(a.q, a.angles, i32(a.pos))[0]
    out, ws = a.run(q_out=a.q)
    assert pc.workspace_status(ws) == 0 and out is a.q
    same(a, a.stored(), want)
    before[:, :, 0] = turned
    assert torch.equal(a.fused, before)


def test_queries_in_place_beside_a_cache_of_4_bits():
    a = Append([60, 9], [20, 3], 16, BF16, FP4, seed=7, given=True)
    want, turned = a.want(), pc.rope(a.q, a.angles, i32(a.pos))[0]
    out, ws = a.run(q_out=a.q)
    assert pc.workspace_status(ws) == 0 and torch.equal(a.q, turned)
    same(a, a.stored(), want)


def test_4_bit_rows_left_out_above_what_one_workgroup_looks_at():
    a = Append([33000, 5, 900], [32990, 1, 800], 64, F16, FP4, heads=1, kvh=1, dim=32, given=True, seed=3)
    a.pos[[0, 32990, 33790]] = a.n_pos
    want = a.want(lost={0, 32990, 33790})
    _, ws = a.run()
    assert pc.workspace_status(ws) == 2
    same(a, a.stored(), want)


@pytest.mark.parametrize("cache", [BF16, FP8, FP4], ids=["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("what", ["nothing", "page", "slot", "table", "position", "offsets"])
def test_rows_left_out_leave_codes_and_scales(cache, what):
    """A row without a page, a slot, or a position of the table: what its slot held stays as it was."""
    a = Append([40, 20, 5], [3, 2, 5], 16, BF16, cache, seed=2, given=what == "position")
    lost = set()
    if what == "page":
        a.table[1], lost = 1 << 20, {3, 4}
    elif what == "slot":
        a.kv[2], a.pos[5:], lost = 3, a.pos[5:] - 2, {5, 6}
    elif what == "table":
        a.angles, a.n_pos, lost = a.angles[:39], 39, {2}
    elif what == "position":
        a.pos[[2, 7]], lost = [a.n_pos, -1], {2, 7}
    elif what == "offsets":     # the second sequence's end is past the rows: it counts as having none, and so does the third
        a.off, lost = [0, 3, 11, 10], set(range(3, 10))
    if what == "offsets":
        off, a.off = a.off, [0, 3, 5, 10]
        want = a.want(lost=lost)
        a.off = off
    else:
        want = a.want(lost=lost)
    _, ws = a.run()
    assert pc.workspace_status(ws) == (2 if lost else 0)
    same(a, a.stored(), want)


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("given", [False, True], ids=["in order", "positions"])
def test_rows_past_32_bits(interleaved, given):
    """Rows 4 GiB apart, and heads 4 GiB apart, on the way in and on the way out."""
    n = (1 << 31) + 4096                                    # elements from one to the next
    table, pos = turn_plain.angles(40, 48), i32([31, 7]) if given else None
    x = rows((2, 3, 64), BF16, torch.Generator().manual_seed(1))
    want = pc.rope(x, table, pos, interleaved=interleaved)[0]
    room = [torch.empty(2 * n, dtype=BF16, device="cuda") for _ in range(2)]
    a, b = (y.as_strided((2, 3, 64), (n, 64, 1)) for y in room)
    a.copy_(x)
    assert torch.equal(pc.rope(a, table, pos, interleaved=interleaved, out=b)[0], want)
    assert torch.equal(pc.rope(a, table, pos, interleaved=interleaved, out=a)[0], want)
    a, b = (y.as_strided((2, 2, 64), (64, n, 1)) for y in room)
    a.copy_(x[:, :2])
    assert torch.equal(pc.rope(a, table, pos, interleaved=interleaved, out=b)[0], want[:, :2])


@pytest.mark.parametrize("cache", [BF16, FP8], ids=["bf16", "fp8"])
def test_appends_past_32_bits(cache):
    """Pages past 4 GiB, rows 4 GiB apart."""
    page, kvh, dim, pages = 1024, 4, 128, 4200 if cache == BF16 else 8400
    codes = [torch.empty((pages, kvh, page, dim), dtype=cache, device="cuda") for _ in range(2)]
    assert codes[0].numel() * codes[0].element_size() > 1 << 32
    scales = [torch.full((kvh,), 0.02, device="cuda") for _ in range(2)] if cache == FP8 else [None, None]
    n = (1 << 31) + 4096
    k, v = (torch.empty(2 * n, dtype=BF16, device="cuda").as_strided((2, kvh, dim), (n, dim, 1)) for _ in range(2))
    g = torch.Generator().manual_seed(3)
    for x in (k, v):
        x.copy_(torch.randn((2, kvh, dim), generator=g))
    table = turn_plain.angles(1600, dim)
    small = [torch.zeros((2, kvh, page, dim), dtype=torch.uint8 if cache == FP8 else cache, device="cuda").view(cache) for _ in range(2)]
    far, near = i32([[pages - 1, pages - 2]]), i32([[1, 0]])
    for pages_of, at in ((codes, far), (small, near)):
        _, ws = pc.kv_append_rope(pc.PagedCache(*pages_of, *scales), at, i32([1025]), i32([0, 2]), k, v, table)
        assert pc.workspace_status(ws) == 0
    for x, y in zip(codes, small):
        for p, s, slot in ((pages - 1, 1, 1023), (pages - 2, 0, 0)):
            got, want = x[p, :, slot].view(torch.uint8), y[s, :, slot].view(torch.uint8)
            assert torch.equal(got, want) and bool(want.any())


def test_codes_are_of_the_sum_in_64_bits_rounded_to_32():
    """3 c is halfway between 5, itself halfway between the codes 4 and 6, and the next number of 32 bits.  The
    other product moves the exact sum off that half: past 2^-52 of it 64 bits hold that, below they do not."""
    c = 6990507 * 2.0 ** -22
    assert float(torch.tensor(c)) == c and 3 * 6990507 == 5 * 2 ** 22 + 1
    for small, code in ((2.0 ** -40, 7), (-(2.0 ** -40), 6), (2.0 ** -60, 6), (-(2.0 ** -60), 6), (0.0, 6)):
        table = torch.tensor([[[c, -small]]], dtype=torch.float32).cuda()
        k = torch.zeros((1, 1, 32), dtype=BF16)
        k[0, 0, 0], k[0, 0, 1], k[0, 0, 31] = 3.0, 1.0, 6.0
        codes = torch.zeros((2, 1, 1, 1, 16), dtype=torch.uint8, device="cuda")
        e = torch.zeros((2, 1, 1, 1, 1), dtype=torch.uint8, device="cuda")
        _, ws = pc.kv_append_rope(pc.PagedCache(codes[0].view(FP4), codes[1].view(FP4), e[0], e[1]), i32([[0]]), i32([1]), i32([0, 1]),
                                  k.cuda(), k.cuda(), table)
        assert pc.workspace_status(ws) == 0
        assert int(e[0]) == 127 and int(codes[0, 0, 0, 0, 0]) & 15 == code
