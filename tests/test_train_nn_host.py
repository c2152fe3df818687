"""nn.py on the host: what the layers hand to the library, with the library's calls replaced (no GPU needed)."""

import ctypes

import pytest
import torch

from paper_2107_03356_amd import nn

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The C calls with their arguments, which do nothing; tensors on the CPU are taken."""
    made = []
    monkeypatch.setattr(nn, "_rows", lambda t, what: t)
    monkeypatch.setattr(nn, "_function", lambda name: lambda *args: 0)
    monkeypatch.setattr(nn, "_call", lambda name, device, *args: made.append((name, args, held(name, args))))
    return made


def held(name, args):
    """The values behind the vector `db` of a weight gradient's call, read while the call runs."""
    if name != "mfac_linear_bwd_weight" or not args[14]:
        return None
    return list((ctypes.c_float * args[4]).from_address(args[14]))


# ---------------------------------------------------------------- db of a weight gradient
@pytest.mark.parametrize("db", [torch.zeros(6, dtype=torch.float64), torch.zeros(5), torch.zeros(6, 1), torch.zeros(6, dtype=BF16),
                                torch.zeros(6, device="meta"), None])
def test_weight_gradient_refuses_db_before_any_call(calls, db):
    dz, x, g = torch.zeros(4, 6, dtype=BF16), torch.zeros(4, 8, dtype=BF16), torch.ones(8)
    with pytest.raises(ValueError):
        nn.linear_backward_weight(dz, x, affine=(g, g), db=db)
    assert not calls


def test_weight_gradient_takes_db_of_any_stride(calls):
    dz, x, g = torch.zeros(4, 6, dtype=BF16), torch.zeros(4, 8, dtype=BF16), torch.ones(8)
    column = torch.arange(18.0).view(6, 3)[:, 1]
    for db in (column, torch.full((1,), 2.5).expand(6), column.contiguous()):
        nn.linear_backward_weight(dz, x, affine=(g, g), db=db)
        assert calls.pop()[2] == db.tolist()


# ---------------------------------------------------------------- what the layers keep and form
class Passes:
    """The passes in elementary operations on the CPU, with a record of what was asked of them."""

    def __init__(self):
        self.made = []

    def layer_norm_forward(self, x, weight=None, bias=None, eps=1e-5, pack=False):
        self.made.append("norm+copy" if pack else "norm")
        mean = x.mean(-1, keepdim=True)
        rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + eps)
        xh = (x - mean) * rstd
        y = xh if weight is None else xh * weight
        y = y if bias is None else y + bias
        flat = x.reshape(-1, x.shape[-1])
        return (y, self.copy(xh), rstd.flatten()) if pack else (y, mean.flatten(), rstd.flatten()[:flat.shape[0]])

    def copy(self, x):
        x = x.reshape(-1, x.shape[-1])
        s = torch.full((x.shape[0], -(-x.shape[1] // 32)), 127 - 5, dtype=torch.uint8)
        return nn.Packed8(torch.round(x * 32).clamp(-127, 127).to(torch.int8), s)

    def value(self, p):
        return p.q.float() / 32 if isinstance(p, nn.Packed8) else p

    def pack8(self, x):
        self.made.append("pack8")
        return self.copy(x)

    def unpack8(self, p, dtype=torch.float32):
        self.made.append("unpack8")
        return self.value(p).to(dtype)

    def linear_forward(self, x, weight, bias=None, act="none", residual=None, keep=None):
        self.made.append("linear" if keep is None else "linear+" + keep)
        z = x @ weight.t() if bias is None else x @ weight.t() + bias
        y = z if act == "none" else torch.nn.functional.silu(z)
        y = y if residual is None else y + residual.reshape(y.shape)
        return y if keep is None else (y, z if keep == "z" else self.copy(z))

    def act_backward(self, dy, z=None, act="none", want_a=False, want_db=True):
        if (z is None) != (act == "none") or (want_a and z is None):
            raise ValueError("act: z goes with an activation")
        self.made.append("act" + "+a" * want_a + "+db" * want_db)
        if z is None:
            return dy, None, dy.reshape(-1, dy.shape[-1]).sum(0) if want_db else None
        v = self.value(z).reshape(dy.shape)
        p = torch.sigmoid(v)
        dz = dy * p * (1 + v * (1 - p))
        return dz, v * p if want_a else None, dz.reshape(-1, dz.shape[-1]).sum(0) if want_db else None

    def linear_backward_input(self, dz, weight, add=None):
        self.made.append("dx")
        return dz @ weight

    def linear_backward_weight(self, dz, x, affine=None, db=None, grad_dtype=None):
        self.made.append("dw")
        x = self.value(x)
        if affine is not None:
            x = x * affine[0] + affine[1]
        return dz.reshape(-1, dz.shape[-1]).t() @ x.reshape(-1, x.shape[-1])

    def layer_norm_backward(self, dy, x, mean, rstd, weight=None, add=None, params=True):
        self.made.append("norm_bwd" + "+params" * params)
        r = rstd.view(*dy.shape[:-1], 1)
        xh = self.value(x).reshape(dy.shape) if isinstance(x, nn.Packed8) else (x - mean.view(r.shape)) * r
        h = dy if weight is None else dy * weight
        dx = r * (h - h.mean(-1, keepdim=True) - xh * (h * xh).mean(-1, keepdim=True))
        dx = dx if add is None else dx + add
        n = dy.shape[-1]
        return (dx, (dy * xh).reshape(-1, n).sum(0), dy.reshape(-1, n).sum(0)) if params else (dx, None, None)


@pytest.fixture
def passes(monkeypatch):
    p = Passes()
    for name in ("layer_norm_forward", "pack8", "unpack8", "linear_forward", "act_backward", "linear_backward_input",
                 "linear_backward_weight", "layer_norm_backward"):
        monkeypatch.setattr(nn, name, getattr(p, name))
    return p


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("copy8", [False, True])
def test_linear_whose_residual_alone_needs_a_gradient(passes, act, copy8):
    x, w, b, r = torch.randn(5, 8), torch.randn(6, 8), torch.randn(6), torch.randn(5, 6, requires_grad=True)
    y = nn.linear(x, w, b, act=act, residual=r, copy8=copy8)
    assert passes.made == ["linear"]
    dy = torch.randn(5, 6)
    y.backward(dy)
    assert torch.equal(r.grad, dy) and passes.made == ["linear"]


@pytest.mark.parametrize("shape", [(20, 6), (2, 10, 6), (4, 5, 6)])
def test_gradient_of_a_residual_of_other_dimensions(passes, shape):
    x, w, r = torch.randn(4, 5, 8), torch.randn(6, 8), torch.randn(*shape, requires_grad=True)
    dy = torch.randn(4, 5, 6)
    nn.linear(x, w, residual=r).backward(dy)
    assert torch.equal(r.grad, dy.view(shape))


@pytest.mark.parametrize("shape", [(8,), (2, 3, 8), ()])
def test_a_weight_is_a_matrix(calls, monkeypatch, shape):
    monkeypatch.setattr(nn, "_rows", lambda t, what: t.reshape(-1, t.shape[-1]) if t.dim() else t.reshape(1, 1))
    x, w = torch.zeros(4, 8), torch.zeros(shape)
    for f in (lambda: nn.linear_forward(x, w), lambda: nn.linear(x, w), lambda: nn.linear_backward_input(torch.zeros(4, 6), w)):
        with pytest.raises(ValueError):
            f()
    assert not calls


def modules(copy8):
    torch.manual_seed(1)
    return nn.LayerNorm(64, copy8=copy8), nn.Linear(64, 64, act="silu", copy8=copy8), nn.FeedForward(64, 32, act="silu", copy8=copy8)


@pytest.mark.parametrize("copy8", [False, True])
@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_inference_keeps_nothing(passes, mode, copy8):
    norm, lin, block = modules(copy8)
    x = torch.randn(3, 4, 64)
    trained = [m(x).detach() for m in (norm, lin, block)]
    del passes.made[:]
    with mode():
        assert torch.equal(norm(x), trained[0]) and passes.made == ["norm"]
        assert torch.equal(lin(x), trained[1]) and passes.made[1:] == ["linear"]
        assert torch.equal(block(x), trained[2]) and passes.made[2:] == ["norm", "linear", "linear"]


@pytest.mark.parametrize("copy8", [False, True])
def test_layers_without_gradients_keep_nothing(passes, copy8):
    norm, lin, block = (m.requires_grad_(False) for m in modules(copy8))
    x = torch.randn(3, 64)
    norm(x), lin(x), block(x)
    assert passes.made == ["norm", "linear", "norm", "linear", "linear"]
    saved = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: saved.append(t) or t, lambda t: t):
        lin(x, residual=torch.randn(3, 64, requires_grad=True))
    assert not saved


def test_training_keeps_what_it_did(passes):
    x = torch.randn(3, 64, requires_grad=True)
    for copy8, want in ((False, ["norm", "linear+z", "norm", "linear+z", "linear"]),
                        (True, ["norm+copy", "linear+pack8", "pack8", "norm+copy", "linear+pack8", "linear"])):
        del passes.made[:]
        for m in modules(copy8):
            m(x)
        assert passes.made == want


NAMES = ["x", "lw", "lb", "w1", "b1", "w2", "b2"]


def block_gradients(needed, copy8):
    torch.manual_seed(4)
    t = [torch.randn(5, 64), 1 + 0.1 * torch.randn(64), torch.randn(64), torch.randn(32, 64) / 8, torch.randn(32),
         torch.randn(64, 32) / 6, torch.randn(64)]
    for name, v in zip(NAMES, t):
        v.requires_grad_(name in needed)
    saved = []
    with torch.autograd.graph.saved_tensors_hooks(lambda v: saved.append(v) or v, lambda v: v):
        y = nn.feed_forward(*t, act="silu", copy8=copy8)
    y.backward(torch.linspace(-1, 1, y.numel()).view(y.shape))
    return {name: v.grad for name, v in zip(NAMES, t) if v.grad is not None}, saved


@pytest.mark.parametrize("copy8", [False, True])
@pytest.mark.parametrize("needed,products", [
    (["x"], ["dx", "dx"]), (["b2"], []), (["w2"], ["dw"]), (["w2", "b2"], ["dw"]), (["b1"], ["dx"]), (["w1"], ["dx", "dw"]),
    (["lw", "lb"], ["dx", "dx"]), (["w1", "w2"], ["dx", "dw", "dw"]), (["x", "b1", "b2"], ["dx", "dx"]),
    (NAMES[1:], ["dx", "dx", "dw", "dw"]), (NAMES, ["dx", "dx", "dw", "dw"])])
def test_block_forms_the_gradients_that_are_needed(passes, needed, products, copy8):
    every, _ = block_gradients(NAMES, copy8)
    del passes.made[:]
    some, saved = block_gradients(needed, copy8)
    assert sorted(some) == sorted(needed)
    for name in needed:
        torch.testing.assert_close(some[name], every[name])
    assert sorted(m for m in passes.made if m in ("dx", "dw")) == sorted(products)
    assert any(m.startswith("norm_bwd") for m in passes.made) == any(n in needed for n in NAMES[:3])
    if needed == ["b2"]:
        assert not saved and passes.made == ["norm", "linear", "linear", "act+db"]


def test_block_refuses_a_missing_parameter_in_training_and_inference(passes):
    t = [torch.randn(5, 64), torch.ones(64), torch.zeros(64), torch.randn(32, 64), torch.zeros(32), torch.randn(64, 32),
         torch.zeros(64)]
    for grad in (True, False):
        for i in range(1, 7):
            with torch.set_grad_enabled(grad), pytest.raises(ValueError):
                nn.feed_forward(*[v if j != i else None for j, v in enumerate(t)])
    assert not passes.made
