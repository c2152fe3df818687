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
