"""The operators over a paged cache at the ends of their arguments' ranges."""
import pytest
import torch

from test_attn_gpu import BF16, F16, FP8, Case

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
