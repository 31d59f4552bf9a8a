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
