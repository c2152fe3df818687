"""The training operators where arguments, values and sizes are out of the ordinary."""

import pytest
import torch

from gpu_common import require_gpu, say
from train_ref import E32, TINY, U, act64, act_error, growth, off, pack64, unpack64  # noqa: F401

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def rand(dev, seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale).to(dev)


def holds(got, want, bound, what):
    o = off(got, want, bound)
    assert o <= 1, (what, o)


# ---------------------------------------------------------------- arguments
def test_weight_gradient_with_db_of_any_stride(dev):
    from paper_2107_03356_amd import nn
    say("db strides")
    dz, p = rand(dev, 1, 50, 40).to(BF16), nn.pack8(rand(dev, 2, 50, 64).to(BF16))
    g, b = rand(dev, 3, 64).to(F32), rand(dev, 4, 64).to(F32)
    _, _, db = nn.act_backward(dz)
    wide = torch.full((40, 3), float("nan"), device=dev)
    wide[:, 1] = db
    want = nn.linear_backward_weight(dz, p, (g, b), db)
    assert torch.equal(nn.linear_backward_weight(dz, p, (g, b), wide[:, 1]), want)
    for bad in (db.cpu(), db.double(), db[:39], None):
        with pytest.raises(ValueError):
            nn.linear_backward_weight(dz, p, (g, b), bad)
