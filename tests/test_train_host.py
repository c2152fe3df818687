"""The training operators' C calls on the host: sizes, and arguments refused before anything is enqueued (no GPU needed)."""

import os

import pytest

from paper_2107_03356_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmfac.so not built")

P = 1 << 20   # an address that nothing reads: every call below returns before it would


def test_workspace_queries():
    lib = B.load()
    assert lib.mfac_layer_norm_bwd_workspace_bytes(-1, 4) == 0
    assert lib.mfac_layer_norm_bwd_workspace_bytes(8, 0) == 0
    assert lib.mfac_layer_norm_bwd_workspace_bytes(0, 100) >= 800
    assert lib.mfac_act_bwd_workspace_bytes(1000, 100) >= 400
    assert lib.mfac_act_bwd_workspace_bytes(1 << 31, 100) == 0
    q = lib.mfac_linear_workspace_bytes
    assert q(B.MFAC_BF16, 0, 64, 64, P, 64, P, 64) == 0
    assert q(7, 8, 64, 64, P, 64, P, 64) == 0
    assert q(B.MFAC_BF16, 8192, 2048, 8192, P, 2048, P, 2048) == 0          # taken as they are, one part of K
    odd = q(B.MFAC_BF16, 8192, 2047, 8192, P, 2047, P, 2047)                # rows not 16-byte aligned: laid out
    assert odd >= 2 * 2048 * (8192 + 8192)
    assert q(B.MFAC_BF16, 8192, 2048, 8192, P + 2, 2048, P, 2048) >= 2 * 2048 * 8192
    assert q(B.MFAC_F32, 8192, 2048, 8192, P, 2048, P, 2048) >= 3 * 2 * 2048 * (8192 + 8192)
    w = lib.mfac_linear_bwd_weight_workspace_bytes
    assert w(B.MFAC_BF16, 8192, 2048, 8192, P, 8192, None, 0) >= 2 * 2048 * 8192   # an 8-bit copy
    assert w(B.MFAC_BF16, 0, 2048, 8192, P, 8192, None, 0) == 0


def pack(**kw):
    a = dict(type=B.MFAC_BF16, rows=4, cols=64, x=P, ldx=64, q=P, ldq=64, s=P)
    a.update(kw)
    return B.mfac_pack8(a["type"], a["rows"], a["cols"], a["x"], a["ldx"], a["q"], a["ldq"], a["s"], None)


@pytest.mark.parametrize("kw", [dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=0), dict(x=None), dict(x=P + 1),
                                dict(ldx=63), dict(q=None), dict(s=None), dict(ldq=63), dict(cols=1 << 31)])
def test_pack8_refuses(kw):
    assert pack(**kw) == B.MFAC_EINVAL


def norm(**kw):
    a = dict(type=B.MFAC_BF16, wtype=B.MFAC_F32, rows=4, cols=64, x=P, ldx=64, w=P, b=P, eps=1e-5, y=P, ldy=64, mean=P,
             rstd=P, q=None, ldq=0, s=None)
    a.update(kw)
    return B.mfac_layer_norm(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(type=9), dict(wtype=B.MFAC_F16), dict(cols=-3), dict(x=None), dict(y=None), dict(ldy=1),
                                dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(w=P + 2), dict(q=P),
                                dict(q=P, s=P, ldq=8), dict(rstd=P + 1)])
def test_layer_norm_refuses(kw):
    assert norm(**kw) == B.MFAC_EINVAL


def norm_bwd(**kw):
    a = dict(type=B.MFAC_BF16, wtype=B.MFAC_F32, rows=4, cols=64, dy=P, lddy=64, x=P, ldx=64, mean=P, rstd=P, q=None, ldq=0,
             s=None, w=P, add=None, ldadd=0, dx=P, lddx=64, dw=P, db=P, ws=P, wb=1 << 30)
    a.update(kw)
    return B.mfac_layer_norm_bwd(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(rstd=None), B.MFAC_EINVAL), (dict(mean=None), B.MFAC_EINVAL), (dict(x=None), B.MFAC_EINVAL),
    (dict(q=P, s=P, ldq=64), B.MFAC_EINVAL),                      # both x and a copy
    (dict(q=P, s=P, ldq=64, x=None), B.MFAC_EINVAL),              # a copy, and a mean
    (dict(add=P, ldadd=3), B.MFAC_EINVAL), (dict(dx=None), B.MFAC_EINVAL), (dict(ws=P + 64), B.MFAC_EINVAL),
    (dict(wb=8), B.MFAC_EWORKSPACE), (dict(ws=None, wb=0), B.MFAC_EWORKSPACE), (dict(wtype=B.MFAC_F16), B.MFAC_EINVAL),
])
def test_layer_norm_bwd_refuses(kw, want):
    assert norm_bwd(**kw) == want


def linear(**kw):
    a = dict(type=B.MFAC_BF16, btype=B.MFAC_F32, act=B.MFAC_ACT_GELU, rows=64, cin=63, cout=64, x=P, ldx=63, w=P, ldw=63,
             bias=P, res=None, ldres=0, y=P, ldy=64, z=None, ldz=0, q=None, ldq=0, s=None, ws=P, wb=1 << 30)
    a.update(kw)
    return B.mfac_linear(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(act=5), B.MFAC_EINVAL), (dict(act=-1), B.MFAC_EINVAL), (dict(btype=B.MFAC_F16), B.MFAC_EINVAL),
    (dict(ldx=62), B.MFAC_EINVAL), (dict(ldw=1), B.MFAC_EINVAL), (dict(y=None), B.MFAC_EINVAL),
    (dict(z=P, ldz=64, q=P, ldq=64, s=P), B.MFAC_EINVAL),         # both a tensor and a copy of z
    (dict(q=P, ldq=64), B.MFAC_EINVAL), (dict(res=P, ldres=2), B.MFAC_EINVAL), (dict(cin=(1 << 21) + 1, ldx=1 << 22, ldw=1 << 22),
                                                                             B.MFAC_EINVAL),
    (dict(wb=0), B.MFAC_EWORKSPACE), (dict(ws=None), B.MFAC_EINVAL), (dict(rows=-1), B.MFAC_EINVAL),
])
def test_linear_refuses(kw, want):
    assert linear(**kw) == want


def act_bwd(**kw):
    a = dict(type=B.MFAC_BF16, act=B.MFAC_ACT_SILU, rows=4, cols=64, dy=P, lddy=64, z=P, ldz=64, q=None, ldq=0, s=None, dz=P,
             lddz=64, a=None, lda=0, db=P, ws=P, wb=1 << 30)
    a.update(kw)
    return B.mfac_act_bwd(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(z=None), B.MFAC_EINVAL), (dict(q=P, ldq=64, s=P), B.MFAC_EINVAL), (dict(act=B.MFAC_ACT_NONE), B.MFAC_EINVAL),
    (dict(act=B.MFAC_ACT_NONE, z=None, a=P, lda=64), B.MFAC_EINVAL), (dict(dz=None), B.MFAC_EINVAL),
    (dict(wb=0), B.MFAC_EWORKSPACE), (dict(db=P + 2), B.MFAC_EINVAL), (dict(lddz=63), B.MFAC_EINVAL),
])
def test_act_bwd_refuses(kw, want):
    assert act_bwd(**kw) == want


def weight(**kw):
    a = dict(type=B.MFAC_BF16, gtype=B.MFAC_F32, rows=64, cin=64, cout=63, dz=P, lddz=63, x=P, ldx=64, q=None, ldq=0, s=None,
             gamma=None, beta=None, db=None, dw=P, lddw=64, ws=P, wb=1 << 30)
    a.update(kw)
    return B.mfac_linear_bwd_weight(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(gtype=B.MFAC_F16), B.MFAC_EINVAL), (dict(x=None), B.MFAC_EINVAL), (dict(q=P, ldq=64, s=P), B.MFAC_EINVAL),
    (dict(gamma=P), B.MFAC_EINVAL), (dict(gamma=P, beta=P), B.MFAC_EINVAL), (dict(dw=None), B.MFAC_EINVAL),
    (dict(lddw=63), B.MFAC_EINVAL), (dict(wb=0), B.MFAC_EWORKSPACE),
])
def test_linear_bwd_weight_refuses(kw, want):
    assert weight(**kw) == want


def test_linear_bwd_input_refuses_and_no_rows_is_nothing_to_do():
    f = B.mfac_linear_bwd_input
    assert f(B.MFAC_BF16, 64, 64, 63, P, 63, P, 64, None, 0, P, 63, P, 1 << 30, None) == B.MFAC_EINVAL
    assert f(B.MFAC_BF16, 64, 64, 63, P, 63, P, 64, P, 3, P, 64, P, 1 << 30, None) == B.MFAC_EINVAL
    assert f(B.MFAC_BF16, 64, 64, 63, P, 63, P, 64, None, 0, P, 64, P, 0, None) == B.MFAC_EWORKSPACE
    assert f(B.MFAC_BF16, 0, 64, 63, None, 63, P, 64, None, 0, None, 64, None, 0, None) == B.MFAC_OK
    assert pack(rows=0) == norm(rows=0) == linear(rows=0) == B.MFAC_OK
