"""The gated block's references against published and independent results (no GPU needed)."""

import pytest
import torch

from gated_ref import drop_factor, gate_slopes64, philox, residual64, residual_back64



@pytest.mark.parametrize("counter,key,want", [
    # the known answers that the generator's authors publish
    ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
])
def test_philox_known_answers(counter, key, want):
    assert [int(v) for v in philox(counter, key)] == want


def test_drop_factor_rate_and_independence_of_width():
    f = drop_factor(400, 1000, 0.3, (7, -5))
    kept = (f != 0).double().mean().item()
    assert abs(kept - 0.7) < 5 * (0.21 / 4e5) ** 0.5
    assert torch.equal(drop_factor(400, 77, 0.3, (7, -5)), f[:, :77])
    assert not torch.equal(drop_factor(400, 77, 0.3, (7, -4)), f[:, :77])
    assert (drop_factor(3, 9, 1.0, (1, 2)) == 0).all() and (drop_factor(3, 9, 2.0 ** -18, (1, 2)) == 1).all()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_gate_slopes_against_autograd(act):
    from train_ref import act64
    g = torch.Generator().manual_seed(3)
    zg, zu, da = (torch.randn(5, 40, generator=g, dtype=torch.float64) for _ in range(3))
    zg.requires_grad_(), zu.requires_grad_()
    y = act64(act, zg)[0] * zu
    y.backward(da)
    (dg, _), (du, _), (a, _) = gate_slopes64(act, zg.detach(), zu.detach(), da, 0 * da)
    torch.testing.assert_close(dg, zg.grad)
    torch.testing.assert_close(du, zu.grad)
    torch.testing.assert_close(a, y.detach())


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post,pre", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("full", [False, True])
def test_residual_gradients_against_autograd(kind, post, pre, full):
    g = torch.Generator().manual_seed(4)

    def leaf(*shape, at=0.0):
        return (at + torch.randn(*shape, generator=g, dtype=torch.float64)).requires_grad_()

    rows, cols, scale, eps = 6, 24, 0.7, 1e-5
    y, r, gate = leaf(rows, cols), leaf(rows, cols), leaf(*((rows, cols) if full else (cols,)), at=0.5)
    w1, b1, w2, b2 = leaf(cols, at=1), leaf(cols), leaf(cols, at=1), leaf(cols)
    zero = torch.zeros(cols, dtype=torch.float64)
    factor = drop_factor(rows, cols, 0.25, (11, 12))
    one, two = ((w1, b1 if kind == "layer" else zero), (w2, b2 if kind == "layer" else zero))
    o = residual64(y, r, one if post else None, two if pre else None, gate, scale, factor, kind, eps)
    ds, dh = (torch.randn(rows, cols, generator=g, dtype=torch.float64) for _ in range(2))
    loss = (o["s"][0] * ds).sum() + ((o["h"][0] * dh).sum() if pre else 0)
    loss.backward()
    d = lambda t: t.detach() if isinstance(t, torch.Tensor) else t   # noqa: E731
    stats = [d(o.get(k, 0.0)) for k in ("mean1", "rstd1", "mean2", "rstd2")]
    b = residual_back64(ds, dh if pre else None, d(y), d(o["s"][0]), stats, tuple(map(d, one)) if post else None,
                        tuple(map(d, two)) if pre else None, d(gate), full, scale, factor, kind)
    wanted = [("dy", y), ("dr", r), ("dgate", gate)]
    wanted += [("dpost_w", w1)] * post + [("dpre_w", w2)] * pre
    if kind == "layer":
        wanted += [("dpost_b", b1)] * post + [("dpre_b", b2)] * pre
    for name, t in wanted:
        torch.testing.assert_close(b[name][0], t.grad)
