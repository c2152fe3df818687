"""Blocks that keep 8-bit copies: the norm's copy of a block's input serves the block's own weight gradient too."""

import pytest
import torch

from gpu_common import require_gpu, say
from test_gpu_gated_ops import rand

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def kept_bytes(f, dtypes=(torch.int8, torch.uint8)):
    """Bytes of the tensors of these types that f keeps for its backward pass, each storage once."""
    seen = {}

    def hook(t):
        if t is not None and t.dtype in dtypes:
            s = t.untyped_storage()
            seen[s.data_ptr()] = s.nbytes()
        return t

    with torch.autograd.graph.saved_tensors_hooks(hook, lambda t: t):
        out = f()
    total = sum(seen.values())
    del out
    return total


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dim", [512, 500])
def test_a_block_keeps_one_copy_of_its_input(dev, kind, dim):
    from paper_2107_03356_amd import nn
    say("one copy of a block's input", kind, dim)
    rows, hid, depth = 1000, 768, 3
    net = nn.GatedStack(dim, hid, depth, kind=kind, copy8=True, device=dev)
    x = rand(dev, 1, rows, dim, dtype=BF16).requires_grad_()
    groups = -(-dim // 32)
    norm, pair = rows * 33 * groups, 2 * rows * 33 * (hid // 32)
    assert kept_bytes(lambda: net(x)) == depth * (norm + pair) + norm   # the last norm's
    assert kept_bytes(lambda: net.blocks[0](x)) == norm + pair
    # where the norm keeps none (nothing before the products is trained), the block makes its own
    for block in net.blocks:
        for v in block.norm.parameters():
            v.requires_grad_(False)
    assert kept_bytes(lambda: net.blocks[0](x.detach())) == norm + pair


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("bias", [False, True])
def test_its_gradients_are_those_of_the_passes(dev, kind, dtype, bias):
    """By hand: the norm with its copy, the layer with its own, and the backward pass with the norm's weight and bias."""
    from paper_2107_03356_amd import nn
    say("gradients of the passes", kind, dtype, bias)
    torch.manual_seed(4)
    rows, dim, hid = 130, 72, 200
    block = nn.GatedFeedForward(dim, hid, kind=kind, bias=bias, copy8=True, device=dev)
    for v in block.norm.parameters():
        torch.nn.init.normal_(v, 1.0, 0.2)
    x, dy = rand(dev, 1, rows, dim, dtype=dtype).requires_grad_(), rand(dev, 2, rows, dim, dtype=dtype)
    block(x).backward(dy)
    w, b = block.norm.weight.detach(), None if kind == "rms" else block.norm.bias.detach()
    up, down = (m.weight.detach().to(dtype) for m in (block.up, block.down))
    o = nn.residual_norm_forward(x.detach(), pre=(w, b), kind=kind, pack=True)
    _, z = nn.gated_linear_forward(o.h, up, None if not bias else block.up.bias.detach(), "silu", keep="pack8")
    dh, dw1, db1, dw2, db2 = nn.gated_feed_forward_backward(dy, o.copy, up, down, z, affine=(w, b), grad_dtype=torch.float32,
                                                            need=(True, True, bias, True, bias))
    g = nn.residual_norm_backward(None, dh, None, o.copy, None, o.pre, pre=(w, b), kind=kind)
    assert torch.equal(block.up.weight.grad, dw1) and torch.equal(block.down.weight.grad, dw2)
    assert torch.equal(block.norm.weight.grad, g.dpre[0]) and (kind == "rms" or torch.equal(block.norm.bias.grad, g.dpre[1]))
    assert torch.equal(x.grad, g.dy + dy)
    if bias:
        assert torch.equal(block.up.bias.grad, db1) and torch.equal(block.down.bias.grad, db2)


def test_rows_without_unit_stride_are_copied_once(dev):
    """Each input that has none is copied for the call, and not a second time to look at it."""
    from paper_2107_03356_amd import nn
    say("copied once")
    rows, cols = 200, 320
    y, r, g = (rand(dev, s, cols, rows).t() for s in (1, 2, 3))
    w = rand(dev, 4, cols, at=1)

    def allocations(*t):
        with torch.no_grad():
            torch.cuda.synchronize()
            before = torch.cuda.memory_stats()["allocation.all.allocated"]
            out = nn.residual_norm(t[0], t[1], pre=(w, None), gate=t[2])
            return torch.cuda.memory_stats()["allocation.all.allocated"] - before, out

    plain, want = allocations(*(t.contiguous() for t in (y, r, g)))
    strided, got = allocations(y, r, g)
    assert strided == plain + 3
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refused_calls_of_residual_norm(dev):
    from paper_2107_03356_amd import nn
    say("refused")
    x, w = rand(dev, 1, 5, 64), rand(dev, 2, 64)
    for kw in (dict(kind="mean"), dict(pre=(w[:63], None)), dict(pre=w), dict(pre=(w, w)), dict(gate=w[:63]), dict(gate=x[:4]),
               dict(residual=x[:4]), dict(p=1.5), dict(p=float("nan")), dict(pre=(w, None), residual=x.half())):
        with pytest.raises(ValueError):
            nn.residual_norm(x, **{**dict(residual=x), **kw})
    with pytest.raises(ValueError):
        nn.residual_norm(x.cpu(), x.cpu())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_captured_and_checkpointed_steps_share_the_copy(dev, kind):
    """A training step of blocks with copy8, captured and replayed, and with its blocks checkpointed."""
    from torch.utils.checkpoint import checkpoint

    from paper_2107_03356_amd import nn
    say("captured step with copies", kind)
    torch.manual_seed(7)
    net = nn.GatedStack(72, 136, 2, kind=kind, copy8=True, post_norm=True, device=dev)
    x, dy = rand(dev, 1, 40, 72, dtype=BF16), rand(dev, 2, 40, 72, dtype=BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            net(x).backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    for v in net.parameters():
        v.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = net(x)
        y.backward(dy)
    again = nn.GatedStack(72, 136, 2, kind=kind, copy8=True, post_norm=True, device=dev)
    again.load_state_dict(net.state_dict())
    for turn in range(3):
        x.copy_(rand(dev, 10 + turn, 40, 72))
        graph.replay()
        torch.cuda.synchronize()
        for v in again.parameters():
            v.grad = None
        want = again(x)
        want.backward(dy)
        assert torch.equal(y, want)
        assert all(torch.equal(v.grad, u.grad) for v, u in zip(net.parameters(), again.parameters()))
    block = again.blocks[0]
    grads = []
    for reentrant in (None, True, False):
        leaf = x.clone().requires_grad_()
        for v in block.parameters():
            v.grad = None
        out = block(leaf) if reentrant is None else checkpoint(block, leaf, use_reentrant=reentrant)
        out.backward(dy)
        grads.append([leaf.grad] + [v.grad for v in block.parameters()])
    assert all(torch.equal(a, b) for other in grads[1:] for a, b in zip(grads[0], other))
