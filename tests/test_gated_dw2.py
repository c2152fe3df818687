"""The second layer's gradient alone: what it takes, on the host (no GPU needed)."""

import os

import pytest
import torch

from paper_2107_03356_amd import _binding as B
from paper_2107_03356_amd import nn

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmfac.so not built")

P = 1 << 20   # an address that nothing reads


def call(**kw):
    a = dict(type=B.MFAC_F32, gtype=B.MFAC_F32, act=B.MFAC_ACT_SILU, rows=1000, cin=48, hidden=400, cout=56, dy=P, lddy=56, w2=None,
             ldw2=0, x=None, ldx=0, q=None, ldq=0, s=None, gamma=None, beta=None, w1=None, ldw1=0, zg=P, zu=P, ldz=800, qg=None, sg=None,
             qu=None, su=None, ldqz=0, dx=None, lddx=0, dw1=None, lddw1=0, db1=None, dw2=P, lddw2=400, ws=P, wb=0)
    a.update(kw)
    return B.mfac_gated_bwd(*a.values(), None)


def test_w2_is_needed_for_the_others_alone():
    assert call() == B.MFAC_EWORKSPACE   # all that is missing
    for other in (dict(dx=P, lddx=48, w1=P, ldw1=48), dict(dw1=P, lddw1=48, x=P, ldx=48), dict(db1=P)):
        assert call(**other) == B.MFAC_EINVAL and call(**other, w2=P, ldw2=400) == B.MFAC_EWORKSPACE


def test_workspace_of_dw2_alone_has_no_da():
    need = B.load().mfac_gated_bwd_workspace_bytes
    rows, hidden, cout = 1000, 4096, 520
    f = lambda type, wanted: need(type, type, rows, 64, hidden, cout, P, cout, P, hidden, P, 64, P, 64, wanted)   # noqa: E731
    product = B.load().mfac_linear_bwd_weight_workspace_bytes
    # dy and a, of fp32 in three 16-bit parts each, and the product's own room (of operands that are laid out: parts of K)
    laid_out = 6 * rows * (cout + hidden)
    assert f(B.MFAC_F32, B.MFAC_GATED_DW2) <= laid_out + product(B.MFAC_F32, rows, hidden, cout, P, cout, P, hidden) - laid_out + 1024
    assert f(B.MFAC_BF16, B.MFAC_GATED_DW2) <= 2 * rows * hidden + product(B.MFAC_BF16, rows, hidden, cout, P, cout, P, hidden) + 1024


def test_nn_takes_no_w2_where_dw2_is_wanted_alone(monkeypatch):
    made = []
    monkeypatch.setattr(nn, "_rows", lambda t, what: t.reshape(-1, t.shape[-1]))
    monkeypatch.setattr(nn, "_function", lambda name: lambda *args: 0)
    monkeypatch.setattr(nn, "_call", lambda name, device, *args: made.append(name))
    dy, z = torch.zeros(5, 16), (torch.zeros(5, 12), torch.zeros(5, 12))
    got = nn.gated_feed_forward_backward(dy, None, None, None, z, need=(False, False, False, True, False))
    assert made == ["mfac_gated_bwd"] and got[3].shape == (16, 12)
    for need in ((True, False, False, True, False), (False, True, False, False, False), (False, False, True, False, False)):
        with pytest.raises(ValueError):
            nn.gated_feed_forward_backward(dy, dy, torch.zeros(24, 16), None, z, need=need)
    with pytest.raises(ValueError):
        nn.gated_feed_forward_backward(dy, None, None, None, None, need=(False, False, False, True, False))
    assert len(made) == 1
