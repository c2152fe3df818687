"""Blocks whose parts a program replaces."""

import pytest
import torch

from gpu_common import require_gpu, say
from test_gpu_gated_ops import rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


@pytest.mark.parametrize("copy8", [False, True])
def test_blocks_with_replaced_parts(dev, copy8):
    """inner and join are called as they are without copies, and with what the norm keeps where there are."""
    from paper_2107_03356_amd import nn
    say("replaced parts", copy8)
    seen = []

    class Block(nn.GatedFeedForward):
        def inner(self, h, *copy):
            seen.append(("inner", len(copy)))
            return super().inner(h, *copy)

        def join(self, y, x, pre=None, **kw):
            seen.append(("join", len(kw)))
            return super().join(y, x, pre, **kw)

    torch.manual_seed(1)
    net = nn.GatedStack(64, 96, 2, copy8=copy8, device=dev)
    x = rand(dev, 1, 30, 64)
    want, alone = net(x), net.blocks[0](x)
    for block in net.blocks:
        block.__class__ = Block
    assert torch.equal(net(x), want)
    assert seen == [("inner", int(copy8)), ("join", int(copy8))] * 2
    seen.clear()
    assert torch.equal(net.blocks[0](x), alone) and seen == [("inner", int(copy8)), ("join", 0)]
    seen.clear()
    with torch.no_grad():   # nothing is kept
        assert torch.equal(net.blocks[0](x), alone) and seen == [("inner", 0), ("join", 0)]
