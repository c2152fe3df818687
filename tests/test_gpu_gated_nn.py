"""Gated blocks with autograd: gradients against the definition in 64 bits and against differences, captured graphs, other
streams, what is kept, and a run of the operators together."""

import pytest
import torch

from gated_ref import drop_factor
from gpu_common import require_gpu, say
from train_ref import U, act64

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


def rand(dev, seed, *shape, scale=1.0, at=0.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return at + scale * torch.randn(*shape, generator=g, device=dev)


def norm64(x, w, b, kind, eps):
    x = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w
    return y if b is None else y + b


def stack64(net, x, factors):
    """A GatedStack's definition on 64-bit copies of its parameters: (output, the copies by name). factors: the blocks'
    dropout, as what each element is multiplied by."""
    p = {n: v.detach().double().requires_grad_() for n, v in net.named_parameters()}
    kind, eps = net.blocks[0].kind, net.blocks[0].eps

    def norm(v, name):
        return norm64(v, p[name + ".weight"], p.get(name + ".bias"), kind, eps)

    s = x
    for i, block in enumerate(net.blocks):
        at = f"blocks.{i}."
        h = norm(s, at + "norm")
        w = p[at + "up.weight"]
        z = h @ w.t()
        if block.up.bias is not None:
            z = z + p[at + "up.bias"]
        zg, zu = z.chunk(2, -1)
        y = (act64(block.up.act, zg)[0] * zu) @ p[at + "down.weight"].t()
        if block.down.bias is not None:
            y = y + p[at + "down.bias"]
        if block.post is not None:
            y = norm(y, at + "post")
        if block.gate is not None:
            y = y * p[at + "gate"]
        s = block.scale * s + y * factors[i]
    return norm(s, "norm"), p


def rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


CONFIGS = [dict(), dict(kind="layer", bias=True, act="gelu"), dict(post_norm=True, gate=0.7, act="gelu_tanh"),
           dict(p=0.2, gate=0.5, scale=0.9, post_norm=True), dict(kind="layer", post_norm=True, p=0.3, act="relu", bias=True),
           dict(act="none", p=0.1)]


@pytest.mark.parametrize("cfg", CONFIGS)
@pytest.mark.parametrize("copy8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_stack_of_blocks(dev, monkeypatch, dtype, copy8, cfg):
    """Output and every gradient of two blocks. In fp32 without copies they are 64 bits' to 1e-5: some hundred roundings of
    2^-24, as sums of squares. bf16: its roundings, 2^-8 each, a dozen on the way; 8-bit copies: half a step of 127 each.
    relu's slope has a step at 0, which a copy moves: a group's largest value is below 4 sigma, so half a step is at most 4/127
    sigma, within which 0.4 * 4/127 = 1.3% of normal values lie on the side with slope 1 and come out with 0. Of a gradient
    that half of the values carry, that is sqrt(0.013 / 0.5) = 0.16."""
    from paper_2107_03356_amd import nn
    say("stack", dtype, copy8, cfg)
    torch.manual_seed(3)
    dim, hid = 72, 136
    net = nn.GatedStack(dim, hid, 2, device=dev, copy8=copy8, **cfg)
    for v in net.parameters():
        if v.dim() == 1:
            torch.nn.init.normal_(v, 1.0, 0.2)
    x = rand(dev, 1, 3, 40, dim).to(dtype).requires_grad_()
    places = [torch.tensor([5 + i, -7 * i], device=dev) for i in range(2)]
    given = iter(places)
    monkeypatch.setattr(nn, "dropout_at", lambda device: next(given))
    y = net(x)
    p = cfg.get("p", 0.0)
    factors = [drop_factor(120, dim, p, v.tolist()).to(dev).view(3, 40, dim) if p else 1.0 for v in places]
    x64 = x.detach().double().requires_grad_()
    want, params = stack64(net, x64, factors)
    dy = rand(dev, 2, 3, 40, dim).to(dtype)
    y.backward(dy)
    want.backward(dy.double())
    most = (1e-5 if dtype == F32 else 12 * U[BF16]) + (6 / 127 if copy8 else 0)
    most += 0.16 if copy8 and cfg.get("act") == "relu" else 0
    assert y.dtype == dtype and rel(y, want) <= most
    assert x.grad.dtype == dtype and rel(x.grad, x64.grad) <= most
    for name, v in net.named_parameters():
        assert v.grad.dtype == v.dtype and rel(v.grad, params[name].grad) <= most, name


@pytest.mark.parametrize("cfg", CONFIGS[:2])
def test_block_alone_is_a_stack_without_its_last_norm(dev, cfg):
    from paper_2107_03356_amd import nn
    say("block alone", cfg)
    torch.manual_seed(3)
    net = nn.GatedStack(72, 136, 2, device=dev, **cfg)
    x = rand(dev, 1, 50, 72)
    s = net.blocks[1](net.blocks[0](x))
    kind = cfg.get("kind", "rms")
    h = nn.rms_norm(s, net.norm.weight) if kind == "rms" else nn.layer_norm(s, net.norm.weight, net.norm.bias, eps=1e-6)
    # h of the stack is formed from s before it is rounded to fp32
    torch.testing.assert_close(net(x), h, rtol=1e-5, atol=1e-5)


def test_gradients_against_differences(dev):
    """The loss along a random direction of every leaf: the central difference of a step h is off by a sum's roundings over h, and
    by h^2; at h = 2e-3 both are below 1e-3 of the slope here."""
    from paper_2107_03356_amd import nn
    say("differences")
    dim, hid, rows = 40, 64, 30
    at = torch.tensor([4, 4], device=dev)
    leaves = [rand(dev, 1, rows, dim), rand(dev, 2, rows, dim), rand(dev, 3, 2 * hid, dim, scale=dim ** -0.5),
              rand(dev, 4, dim, hid, scale=hid ** -0.5), rand(dev, 5, dim, at=1, scale=0.2), rand(dev, 6, dim, at=1, scale=0.2),
              rand(dev, 7, dim, at=0.5, scale=0.2), rand(dev, 8, rows, dim, at=0.5, scale=0.2), rand(dev, 9, 2 * hid), rand(dev, 10, dim)]
    c1, c2 = rand(dev, 20, rows, dim), rand(dev, 21, rows, dim)

    def loss(v):
        x, r, w1, w2, post, pre, gate, gates, b1, b2 = v
        y = nn.gated_feed_forward(x, w1, w2, b1, b2)
        s, h = nn.residual_norm(y, r, post=(post, None), pre=(pre, None), gate=gate, p=0.2, at=at)
        s2, _ = nn.residual_norm(nn.gated_linear(h, w1[:2 * dim]), s, gate=gates, scale=0.5)
        return (s.double() * c1).sum() + (s2.double() * c2).sum()

    v = [t.clone().requires_grad_() for t in leaves]
    loss(v).backward()
    for i, t in enumerate(leaves):
        d = rand(dev, 100 + i, *t.shape)
        slope = (v[i].grad.double() * d).sum().item()
        h = 2e-3
        ends = [loss([u + s * h * d if j == i else u for j, u in enumerate(leaves)]).item() for s in (1, -1)]
        size = (v[i].grad.double().norm() * d.norm()).item()
        assert abs((ends[0] - ends[1]) / (2 * h) - slope) <= 5e-3 * size, i


@pytest.mark.parametrize("copy8", [False, True])
def test_one_by_one_the_gradients_are_those_of_all(dev, copy8):
    from paper_2107_03356_amd import nn
    say("one by one", copy8)
    at = torch.tensor([4, 4], device=dev)
    dy = rand(dev, 30, 4, 25, 72).to(BF16)
    make = [lambda: rand(dev, 1, 4, 25, 72).to(BF16), lambda: rand(dev, 2, 2 * 136, 72, scale=0.1), lambda: rand(dev, 3, 272),
            lambda: rand(dev, 4, 72, 136, scale=0.1), lambda: rand(dev, 5, 72), lambda: rand(dev, 6, 100, 72).to(BF16),
            lambda: rand(dev, 7, 72, at=1), lambda: rand(dev, 8, 72, at=1), lambda: rand(dev, 9, 72)]

    def gradients(needed):
        t = [f() for f in make]
        for i in needed:
            t[i].requires_grad_()
        x, w1, b1, w2, b2, r, post, pre, gate = t
        y = nn.gated_feed_forward(x, w1, w2, b1, b2, act="gelu", copy8=copy8)
        s, h = nn.residual_norm(y, r, post=(post, None), pre=(pre, None), gate=gate, p=0.1, at=at, copy8=copy8)
        torch.autograd.backward([s, h], [dy, 2 * dy])
        assert [v.grad is not None for v in t] == [i in needed for i in range(len(t))]
        return {i: t[i].grad for i in needed}

    every = gradients(range(9))
    assert every[5].shape == (100, 72)
    for needed in [[i] for i in range(9)] + [[1, 3], [0, 4], [6, 8]]:
        for i, g in gradients(needed).items():
            # without db, dz comes straight from the product that forms da: the same values where hidden is no multiple of 64
            assert torch.equal(g, every[i]), (needed, i)


def test_unused_outputs(dev):
    """s alone, h alone, or neither takes part in the loss."""
    from paper_2107_03356_amd import nn
    say("unused outputs")
    y0, r0, w0 = rand(dev, 1, 20, 64), rand(dev, 2, 20, 64), rand(dev, 3, 64, at=1)
    ds, dh = rand(dev, 4, 20, 64), rand(dev, 5, 20, 64)

    def run(use_s, use_h):
        y, r, w = (t.clone().requires_grad_() for t in (y0, r0, w0))
        s, h = nn.residual_norm(y, r, pre=(w, None))
        torch.autograd.backward([t for t, u in ((s, use_s), (h, use_h)) if u], [t for t, u in ((ds, use_s), (dh, use_h)) if u])
        return y.grad, r.grad, w.grad

    s_only, h_only, both = run(True, False), run(False, True), run(True, True)
    assert torch.equal(s_only[0], ds) and s_only[2] is None
    torch.testing.assert_close(s_only[0] + h_only[0], both[0])
    assert torch.equal(h_only[2], both[2])


def test_inference_keeps_nothing(dev):
    from paper_2107_03356_amd import nn
    say("inference")
    torch.manual_seed(2)
    for copy8 in (False, True):
        net = nn.GatedStack(64, 128, 2, p=0.5, copy8=copy8, device=dev).eval()
        lin, rms, drop = nn.GatedLinear(64, 40, device=dev), nn.RMSNorm(64, device=dev), nn.Dropout(0.5).eval()
        x = rand(dev, 1, 30, 64).to(BF16)
        trained = [m(x).detach() for m in (net, lin, rms, drop)]
        kept = []
        with torch.no_grad(), torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
            assert all(torch.equal(m(x), t) for m, t in zip((net, lin, rms, drop), trained))
        assert not kept


def test_one_token_by_one_is_the_batch(dev):
    """Rows of a batch up to 16 and single tokens run through the same sums."""
    from paper_2107_03356_amd import nn
    say("tokens")
    torch.manual_seed(1)
    for dtype in (F32, BF16):
        lin = nn.GatedLinear(200, 120, bias=True, device=dev)
        x, r, w = rand(dev, 1, 16, 200).to(dtype), rand(dev, 2, 16, 120).to(dtype), rand(dev, 3, 120, at=1)
        with torch.no_grad():
            y = lin(x)
            s, h = nn.residual_norm(y, r, pre=(w, None))
            for i in range(16):
                yi = lin(x[i])
                si, hi = nn.residual_norm(yi, r[i], pre=(w, None))
                assert yi.shape == (120,) and torch.equal(yi, y[i]) and torch.equal(si, s[i]) and torch.equal(hi, h[i])


# ---------------------------------------------------------------- graphs, streams, memory
def test_captured_training_step(dev):
    """A step of the stack with dropout, captured: each replay draws anew, and is what the passes give for what it drew."""
    from paper_2107_03356_amd import nn
    say("graph")
    torch.manual_seed(7)
    net = nn.GatedStack(64, 128, 2, p=0.25, post_norm=True, device=dev)
    x, dy = rand(dev, 1, 40, 64).to(BF16), rand(dev, 2, 40, 64).to(BF16)
    drawn = []
    draw, nn.dropout_at = nn.dropout_at, lambda device: drawn.append(draw(device)) or drawn[-1]
    try:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(2):
                net(x).backward(dy)
        torch.cuda.current_stream().wait_stream(side)
        for v in net.parameters():
            v.grad = None
        drawn.clear()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = net(x)
            y.backward(dy)
        held = list(drawn)
        seen = []
        for turn in range(3):
            x.copy_(rand(dev, 10 + turn, 40, 64))
            graph.replay()
            torch.cuda.synchronize()
            got = y.clone(), [v.grad.clone() for v in net.parameters()]
            places = [t.clone() for t in held]
            seen.append(torch.stack(places))
            again = iter(places)
            nn.dropout_at = lambda device: next(again)
            eager = nn.GatedStack(64, 128, 2, p=0.25, post_norm=True, device=dev)
            eager.load_state_dict(net.state_dict())
            want = eager(x)
            want.backward(dy)
            assert torch.equal(got[0], want)
            for g, v in zip(got[1], eager.parameters()):
                assert torch.equal(g, v.grad)
        assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])
    finally:
        nn.dropout_at = draw


def test_checkpointing_draws_the_same_mask(dev):
    from torch.utils.checkpoint import checkpoint

    from paper_2107_03356_amd import nn
    say("checkpoint")
    block = nn.GatedFeedForward(64, 128, p=0.4, device=dev)
    x = rand(dev, 1, 30, 64)
    grads = []
    for again in (False, True):
        leaf = x.clone().requires_grad_()
        torch.manual_seed(11)
        y = checkpoint(block, leaf, use_reentrant=False) if again else block(leaf)
        y.square().sum().backward()
        grads.append(leaf.grad)
    assert torch.equal(*grads)


def test_two_streams_at_once(dev):
    """Calls on two streams share no workspace."""
    from paper_2107_03356_amd import nn
    say("streams")
    torch.manual_seed(1)
    nets = [nn.GatedStack(128, 264, 1, post_norm=True, device=dev) for _ in range(2)]
    xs = [rand(dev, i, 600, 128).to(BF16) for i in range(2)]
    dys = [rand(dev, 5 + i, 600, 128).to(BF16) for i in range(2)]

    def step(i):
        for v in nets[i].parameters():
            v.grad = None
        y = nets[i](xs[i])
        y.backward(dys[i])
        return [y.detach()] + [v.grad for v in nets[i].parameters()]

    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append(step(i))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_the_same_twice(dev):
    """Sums are joined in a fixed order."""
    from paper_2107_03356_amd import nn
    say("twice")
    x = rand(dev, 1, 3000, 264)
    w1, w2 = rand(dev, 2, 2 * 515, 264, scale=0.06), rand(dev, 3, 264, 515, scale=0.04)
    pre, post, gate = (rand(dev, s, 264, at=1) for s in (4, 5, 6))
    ds, dh = rand(dev, 7, 3000, 264), rand(dev, 8, 3000, 264)
    for dtype in (F32, BF16):
        runs = []
        for _ in range(2):
            t = [v.to(dtype).requires_grad_() for v in (x.clone(), w1.clone(), w2.clone())] + [
                v.clone().requires_grad_() for v in (pre, post, gate)]
            y = nn.gated_feed_forward(t[0], t[1], t[2])
            s, h = nn.residual_norm(y, t[0], pre=(t[3], None), post=(t[4], None), gate=t[5])
            torch.autograd.backward([s, h], [ds.to(dtype), dh.to(dtype)])
            runs.append([s, h] + [v.grad for v in t])
        assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_strides_and_views(dev):
    """Rows that do not lie side by side, transposed and broadcast inputs."""
    from paper_2107_03356_amd import nn
    say("strides")
    base = rand(dev, 1, 20, 3, 64)
    x, r = base[:, 1], rand(dev, 2, 64, 20).t()
    w, gate = rand(dev, 3, 64, at=1), rand(dev, 4, 64)
    weight = rand(dev, 5, 64, 80).t()
    s, h = nn.residual_norm(x, r, pre=(w[::1], None), gate=gate.expand(20, 64))
    s2, h2 = nn.residual_norm(x.contiguous(), r.contiguous(), pre=(w, None), gate=gate)
    torch.testing.assert_close(s, s2)
    torch.testing.assert_close(h, h2)
    assert torch.equal(nn.gated_linear(x, weight), nn.gated_linear(x.contiguous(), weight.contiguous()))
    at = torch.tensor([1, 2], device=dev)
    assert torch.equal(nn.dropout(r, 0.5, at=at), nn.dropout(r.contiguous(), 0.5, at=at))
    # a gate that is broadcast gets the sum of its gradients
    a, b = gate.clone().requires_grad_(), gate.clone().requires_grad_()
    nn.residual_norm(x, r, gate=a.expand(20, 64))[0].sum().backward()
    nn.residual_norm(x, r, gate=b)[0].sum().backward()
    torch.testing.assert_close(a.grad, b.grad, rtol=1e-5, atol=1e-5)


def test_memory_of_dropout_and_copies(dev):
    """A mask is not kept: what dropout keeps is where it starts. With copy8 a block keeps about half of bf16's bytes."""
    from paper_2107_03356_amd import nn
    say("kept bytes")

    def kept(f):
        seen = {}

        def hook(t):
            s = t.untyped_storage()
            seen[s.data_ptr()] = s.nbytes()
            return t

        with torch.autograd.graph.saved_tensors_hooks(hook, lambda t: t):
            out = f()
        del out
        return sum(seen.values())

    x = rand(dev, 1, 4096, 512).to(BF16).requires_grad_()
    assert kept(lambda: nn.dropout(x, 0.1)) <= 512
    w = [rand(dev, 2, 2 * 1024, 512).to(BF16).requires_grad_(), rand(dev, 3, 512, 1024).to(BF16).requires_grad_()]
    weights = sum(v.untyped_storage().nbytes() for v in w)
    whole, small = (kept(lambda: nn.gated_feed_forward(x, *w, copy8=c)) - weights for c in (False, True))
    assert whole == 2 * 4096 * (512 + 2048) and small <= 0.52 * whole, (whole, small)


@pytest.mark.parametrize("args", [["--gated"], ["--gated", "--dropout", "0.1", "--copy8", "--bf16"]])
def test_example_runs(dev, args, monkeypatch, capsys):
    import importlib.util
    import os
    import sys
    say("example", args)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward_mfac.py")
    spec = importlib.util.spec_from_file_location("feed_forward_mfac", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", [path, "--steps", "3", "--rows", "256", "--dim", "72", "--blocks", "2"] + args)
    example.main()
    out = capsys.readouterr().out
    assert "optimizer status 0" in out and "nan" not in out


def test_example_model_gradients(dev):
    """The example's gated model against the definition in 64 bits."""
    import importlib.util
    import os
    say("example gradients")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward_mfac.py")
    spec = importlib.util.spec_from_file_location("feed_forward_mfac", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    torch.manual_seed(0)
    net = example.model(48, 2, False, dev, gated=True)
    x, dy = rand(dev, 1, 64, 48), rand(dev, 2, 64, 48)
    net(x).backward(dy)
    h, p = stack64(net[0], x.double(), [1.0, 1.0])
    w, b = (v.detach().double().requires_grad_() for v in (net[1].weight, net[1].bias))
    (h @ w.t() + b).backward(dy.double())
    for name, v in net[0].named_parameters():
        assert rel(v.grad, p[name].grad) <= 1e-5, name
    assert rel(net[1].weight.grad, w.grad) <= 1e-5
