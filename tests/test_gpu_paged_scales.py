"""Attention over fp8 pages with large V scales: outputs that fp32 holds come out."""

import pytest
import torch

from tests.paged_util import Attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("grid", [(28, 28), (60, 60)])  # whole requests and splits
def test_large_v_scales(grid, out, group):
    """Equal weights over rows of up to 2^125: their sum times the scale is past fp32, their
    mean is not."""
    n = grid[0] * grid[1]
    x = Attend(batch=2, heads=(2 * group, 2), grid=grid, pos=[n - 1, n // 2], kv="fp8", out=out,
               scale=0.0, seed=group)
    x.v_scale.mul_(2.0 ** 123)
    x.v64 *= 2.0 ** 123
    x.run()
    x.check()
    x.v_scale.mul_(2.0 ** -90).mul_(2.0 ** -93)  # 2^-183 is 0 in fp32
    x.v64 *= 2.0 ** -183
    x.run()
    x.check()
    assert torch.isfinite(x.out).all()
