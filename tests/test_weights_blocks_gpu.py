"""The weights that pc_attn_paged adds up for few rows: several blocks of keys, room of any width and alignment, blocks
that a window leaves out, in place or beside, over caches of 16, 8 and 4 bits."""
import pytest
import torch

from test_attn_fp4_gpu import Case4
from test_attn_gpu import BF16, F16, FP8, Case

pytestmark = pytest.mark.gpu

# lengths on both sides of a block of 1,024 keys, an idle sequence, rows that fill no, one and more than eight teams
KV, NEW = [5280, 3000, 1024, 1025, 0, 7, 2048, 1023], [1, 3, 1, 2, 0, 1, 3, 2]


@pytest.fixture(autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("heads,kvh,dtype,cache", [(14, 2, BF16, "fp4"), (10, 1, F16, "fp4"), (14, 2, F16, "own"), (8, 8, BF16, "own"),
                                                   (6, 3, BF16, "fp8")])
@pytest.mark.parametrize("extra,shift", [(0, 0), (4, 0), (1, 0), (2, 2), (0, 1), (3, 3)])
@pytest.mark.parametrize("window", [0, 500])
def test_blocks_of_keys(heads, kvh, dtype, cache, extra, shift, window):
    kw = dict(heads=heads, kvh=kvh, dim=32, page=16, cols=330, dtype=dtype, weights=True, seed=heads + extra)
    c = Case4(KV, NEW, **kw) if cache == "fp4" else Case(KV, NEW, cache=FP8 if cache == "fp8" else dtype, **kw)
    room, plain = c.cols * c.page, c.weight
    n, stride = len(KV), room + extra

    def buffer():   # `shift` floats from a multiple of 16 bytes
        x = torch.full((n * kvh * stride + 4,), -7.0, device="cuda")
        return x, x[shift:shift + n * kvh * stride].view(n, kvh, stride)
    (whole, old), (whole_out, out) = buffer(), buffer()
    old[:, :, :room] = plain

    def run(weight_out):
        c.weight = old
        got = c.run(window=window, weight_out=weight_out, max_kv=room)
        c.weight = plain
        return got
    got = run(out)
    c.check((got[0], got[1], out[:, :, :room], got[3]), window=window)
    beside = out[:, :, :room].clone()
    assert bool((out[:, :, room:] == -7).all()) and bool((whole_out[:shift] == -7).all()) and bool((whole_out[shift + out.numel():] == -7).all())
    assert torch.equal(old[:, :, :room], plain)
    for s in range(n):
        assert not bool(out[s, :, KV[s]:room].any())
        if window and NEW[s]:
            first = max(0, KV[s] - NEW[s] - window + 1)
            assert torch.equal(out[s, :, :first], plain[s, :, :first])
    run(old)
    assert torch.equal(old[:, :, :room], beside)
    assert bool((old[:, :, room:] == -7).all())
