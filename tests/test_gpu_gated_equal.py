"""Layer norm, between two blocks, of rows whose values are all equal."""

import pytest
import torch

from gated_ref import ROW
from gpu_common import require_gpu, say
from test_gpu_gated_ops import rand
from train_ref import E32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


@pytest.mark.parametrize("cols", [7, 300, 1000, 2047, 4093, 8191, 9001, 16383])
@pytest.mark.parametrize("size", [1.0, 1000.0])
def test_rows_of_equal_values(dev, size, cols):
    """What is left of them is the error of their mean: ROW units of 2^-24 of the value, and its division and the difference
    round; times 1 / sqrt(eps) at most. bf16 values have exact sums, and leave nothing."""
    from paper_2107_03356_amd import nn
    say("rows of equal values", size, cols)
    eps = 1e-6
    x = (size * rand(dev, 1, 50, 1)).expand(50, cols).contiguous()
    units = (ROW + 2) * E32 * x.abs().double()
    for residual in (None, 0 * x):
        o = nn.residual_norm_forward(x, residual, pre=(None, None), kind="layer", eps=eps)
        assert (o.h.abs() <= units / eps ** 0.5).all() and ((o.pre[0] - x[:, 0]).abs() <= units[:, 0]).all()
        y, r = x.to(torch.bfloat16), None if residual is None else residual.to(torch.bfloat16)
        o = nn.residual_norm_forward(y, r, pre=(None, None), kind="layer", eps=eps)
        assert (o.h == 0).all() and torch.equal(o.pre[0], y[:, 0].float())
