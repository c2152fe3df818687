"""The gated block's functions of nn.py on the host: what they refuse, with the library's calls replaced (no GPU needed)."""

import pytest
import torch

from paper_2107_03356_amd import nn

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture
def calls(monkeypatch):
    """The C calls with their arguments, which do nothing; tensors on the CPU are taken."""
    made = []
    monkeypatch.setattr(nn, "_rows", lambda t, what: t.reshape(-1, t.shape[-1]))
    monkeypatch.setattr(nn, "_function", lambda name: lambda *args: 0)
    monkeypatch.setattr(nn, "_call", lambda name, device, *args: made.append((name, args)))
    return made


def z(*shape, dtype=BF16, device=None):
    return torch.zeros(*shape, dtype=dtype, device=device)


X, W1, W2 = z(5, 16), z(24, 16), z(16, 12)
PAIR = (z(5, 12), z(5, 12))


@pytest.mark.parametrize("f", [
    lambda: nn.gated_linear_forward(X, z(23, 16)), lambda: nn.gated_linear_forward(X, z(24, 15)),
    lambda: nn.gated_linear_forward(X, z(24, 16, dtype=F32)), lambda: nn.gated_linear_forward(X, W1, act="tanh"),
    lambda: nn.gated_linear_forward(X, W1, keep="y"), lambda: nn.gated_linear_forward(X, W1, z(12)),
    lambda: nn.gated_linear_forward(X, W1, z(24, dtype=F16)), lambda: nn.gated_linear_forward(X, z(16)),
    lambda: nn.gated_linear_forward(X.double(), W1.double()), lambda: nn.gated_linear(X, W1, act="tanh"),
    lambda: nn.gated_linear_backward(PAIR[0], X, W1, PAIR[0]), lambda: nn.gated_linear_backward(PAIR[0], X, W1, (PAIR[0], z(5, 11))),
    lambda: nn.gated_linear_backward(PAIR[0], X, W1, (PAIR[0], z(5, 12, dtype=F32))), lambda: nn.gated_linear_backward(PAIR[0], X, W1, None),
    lambda: nn.gated_linear_backward(PAIR[0], z(4, 16), W1, PAIR), lambda: nn.gated_linear_backward(PAIR[0], X, z(24, 15), PAIR),
    lambda: nn.gated_linear_backward(PAIR[0], z(5, 15), W1, PAIR), lambda: nn.gated_linear_backward(PAIR[0], X, W1, PAIR, grad_dtype=F16),
    lambda: nn.gated_feed_forward_backward(X, X, W1, z(15, 12), PAIR), lambda: nn.gated_feed_forward_backward(X, X, W1, W2, PAIR, "nope"),
    lambda: nn.gated_feed_forward_backward(X, X, W1, W2, PAIR, affine=(z(16, dtype=F32), z(15, dtype=F32))),
    lambda: nn.gated_feed_forward_backward(X, X, W1, W2, PAIR, affine=(None, z(16, dtype=F32))),
    lambda: nn.residual_norm_forward(z(1, 32769), pre=(None, None)), lambda: nn.residual_norm_forward(X, kind="mean"), lambda: nn.residual_norm_forward(X, z(4, 16)),
    lambda: nn.residual_norm_forward(X, z(5, 16, dtype=F32)), lambda: nn.residual_norm_forward(X, pre=(z(16), z(16))),
    lambda: nn.residual_norm_forward(X, pre=z(15)), lambda: nn.residual_norm_forward(X, pre=(z(15), None)),
    lambda: nn.residual_norm_forward(X, pre=(z(16), None), post=(z(16, dtype=F32), None)), lambda: nn.residual_norm_forward(X, X, pack=True),
    lambda: nn.residual_norm_forward(X, gate=z(15)), lambda: nn.residual_norm_forward(X, gate=z(4, 16)),
    lambda: nn.residual_norm_forward(X, gate=z(5, 16, dtype=F32)), lambda: nn.residual_norm_forward(X, X, p=0.5),
    lambda: nn.residual_norm_forward(X, X, p=1.5, at=z(2, dtype=torch.int64)), lambda: nn.residual_norm_forward(X, X, p=0.5, at=z(2)),
    lambda: nn.residual_norm_forward(X, X, p=0.5, at=z(3, dtype=torch.int64)),
    lambda: nn.residual_norm_backward(None, None, X, X), lambda: nn.residual_norm_backward(X, X, X, X),
    lambda: nn.residual_norm_backward(X, None, X, X, pre=(z(16), None)), lambda: nn.residual_norm_backward(X, X, X, X, pre=(z(16), None)),
    lambda: nn.residual_norm_backward(X, X, X, None, None, (None, z(5, dtype=F32)), pre=(z(16), None)),
    lambda: nn.residual_norm_backward(X, X, X, X, None, (None, z(4, dtype=F32)), pre=(z(16), None)),
    lambda: nn.residual_norm_backward(X, X, X, X, None, (None, z(5)), pre=(z(16), None)),
    lambda: nn.residual_norm_backward(X, X, X, X, None, (None, z(5, dtype=F32)), pre=(z(16), z(16)), kind="layer"),
    lambda: nn.residual_norm_backward(X, None, None, X, (None, z(5, dtype=F32)), post=(z(16), None)),
    lambda: nn.residual_norm_backward(X, z(4, 16), X, X, None, (None, z(5, dtype=F32)), pre=(z(16), None)),
    lambda: nn.residual_norm_backward(X, None, None, None, gate=z(16)),
    lambda: nn.dropout_forward(X, 0.5, None), lambda: nn.dropout_forward(X, -0.5, z(2, dtype=torch.int64)),
    lambda: nn.dropout_forward(X, float("nan"), z(2, dtype=torch.int64)), lambda: nn.Dropout(1.5),
    lambda: nn.GatedFeedForward(16, 32, kind="both"), lambda: nn.GatedFeedForward(16, 32, p=2.0), lambda: nn.GatedStack(16, 32, 0),
])
def test_refused_in_words_before_any_call(calls, f):
    with pytest.raises(ValueError):
        f()
    assert not calls


def test_what_is_taken_is_called_once(calls):
    at = z(2, dtype=torch.int64)
    nn.gated_linear_forward(X, W1, keep="z")
    nn.gated_linear_backward(PAIR[0], X, W1, PAIR)
    nn.gated_feed_forward_backward(X, X, W1, W2, PAIR, need=(True, True, True, True, False))
    nn.residual_norm_forward(X, X, post=(z(16), None), pre=(None, None), gate=z(16), p=0.5, at=at, pack=True)
    nn.residual_norm_backward(X, X, X, X, (None, z(5, dtype=F32)), (None, z(5, dtype=F32)), post=(z(16), None), pre=(None, None))
    nn.dropout_forward(X, 0.5, at)
    assert [name for name, _ in calls] == ["mfac_gated_linear", "mfac_gated_bwd", "mfac_gated_bwd", "mfac_residual_norm",
                                           "mfac_residual_norm_bwd", "mfac_dropout"]


def test_nothing_between_is_nothing_done(calls):
    assert nn.residual_norm(X) == (X, None) and nn.residual_norm_forward(X).s is X
    assert nn.dropout(X, 0.0) is X and nn.dropout(X, 0.5, training=False) is X
    assert nn.gated_linear_backward(PAIR[0], X, W1, PAIR, need=(False, False, False)) == (None, None, None)
    assert not calls


def test_needs_decide_what_is_formed(calls):
    w = z(16)
    r = (None, z(5, dtype=F32))
    g = nn.residual_norm_backward(X, X, X, X, r, r, post=(w, None), pre=(w, None), gate=w, need=(False, True, False, True))
    assert g.dy is None and g.dresidual is not None and g.dgate is None and g.dpost[0] is not None and g.dpost[1] is None
    g = nn.residual_norm_backward(X, X, X, X, r, r, post=(w, None), pre=(w, None), gate=w, need=(True, False, True, False))
    assert g.dy is not None and g.dresidual is None and g.dgate.shape == (16,) and g.dpost == g.dpre == (None, None)
    # one gradient serves both where nothing lies between
    g = nn.residual_norm_backward(X, X, None, X, None, r, pre=(w, None))
    assert g.dy is g.dresidual
    g = nn.residual_norm_backward(X, X, None, X, None, r, pre=(w, None), scale=0.5)
    assert g.dy is not g.dresidual
