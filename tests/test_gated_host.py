"""The gated block's C calls on the host: sizes, and arguments refused before anything is enqueued (no GPU needed)."""

import os

import pytest

from paper_2107_03356_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmfac.so not built")

P = 1 << 20   # an address that nothing reads: every call below returns before it would
BIG = 1 << 40
EINVAL, EWORKSPACE, OK = B.MFAC_EINVAL, B.MFAC_EWORKSPACE, B.MFAC_OK
POST, PRE, LAYER = B.MFAC_NORM_POST, B.MFAC_NORM_PRE, B.MFAC_NORM_LAYER


def gated(**kw):
    a = dict(type=B.MFAC_BF16, btype=B.MFAC_F32, act=B.MFAC_ACT_SILU, rows=64, cin=63, hidden=40, x=P, ldx=63, w=P, ldw=63, bias=P,
             y=P, ldy=40, zg=None, zu=None, ldz=0, qg=None, sg=None, qu=None, su=None, ldq=0, ws=P, wb=BIG)
    a.update(kw)
    return B.mfac_gated_linear(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(type=3), EINVAL), (dict(btype=B.MFAC_F16), EINVAL), (dict(act=5), EINVAL), (dict(act=-1), EINVAL), (dict(rows=-1), EINVAL),
    (dict(cin=0), EINVAL), (dict(hidden=0), EINVAL), (dict(hidden=(1 << 20) + 1, ldy=1 << 21), EINVAL), (dict(x=None), EINVAL),
    (dict(w=None), EINVAL), (dict(y=None), EINVAL), (dict(ldx=62), EINVAL), (dict(ldw=62), EINVAL), (dict(ldy=39), EINVAL),
    (dict(x=P + 1), EINVAL), (dict(bias=P + 2), EINVAL), (dict(zg=P), EINVAL), (dict(zu=P, ldz=40), EINVAL),
    (dict(zg=P, zu=P, ldz=39), EINVAL), (dict(qg=P, sg=P, ldq=40), EINVAL), (dict(qg=P, sg=P, qu=P, ldq=40), EINVAL),
    (dict(qg=P, sg=P, qu=P, su=P, ldq=39), EINVAL), (dict(zg=P, zu=P, ldz=40, qg=P, sg=P, qu=P, su=P, ldq=40), EINVAL),
    (dict(wb=0), EWORKSPACE), (dict(ws=None), EINVAL), (dict(ws=P + 8), EINVAL), (dict(rows=0, x=None), OK),
])
def test_gated_linear_refuses(kw, want):
    assert gated(**kw) == want


def backward(**kw):
    a = dict(type=B.MFAC_BF16, gtype=B.MFAC_F32, act=B.MFAC_ACT_SILU, rows=64, cin=48, hidden=40, cout=56, dy=P, lddy=56, w2=P,
             ldw2=40, x=P, ldx=48, q=None, ldq=0, s=None, gamma=None, beta=None, w1=P, ldw1=48, zg=P, zu=P, ldz=80, qg=None, sg=None,
             qu=None, su=None, ldqz=0, dx=P, lddx=48, dw1=P, lddw1=48, db1=P, dw2=P, lddw2=40, ws=P, wb=BIG)
    a.update(kw)
    return B.mfac_gated_bwd(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(type=-1), EINVAL), (dict(gtype=B.MFAC_F16), EINVAL), (dict(act=9), EINVAL), (dict(rows=-1), EINVAL), (dict(cin=0), EINVAL),
    (dict(hidden=0), EINVAL), (dict(cout=-1), EINVAL), (dict(cout=(1 << 21) + 1), EINVAL), (dict(dy=None), EINVAL), (dict(lddy=55), EINVAL),
    (dict(w2=None), EINVAL), (dict(ldw2=39), EINVAL), (dict(cout=0), EINVAL), (dict(cout=0, dw2=None, lddy=39), EINVAL),
    (dict(x=None), EINVAL), (dict(x=None, q=P, ldq=48), EINVAL), (dict(q=P, ldq=48, s=P), EINVAL), (dict(x=None, q=P, ldq=47, s=P), EINVAL),
    (dict(beta=P), EINVAL), (dict(gamma=P + 1), EINVAL), (dict(w1=None), EINVAL), (dict(ldw1=47), EINVAL), (dict(zg=None), EINVAL),
    (dict(zg=None, zu=None), EINVAL), (dict(ldz=39), EINVAL), (dict(qg=P, sg=P, qu=P, su=P, ldqz=40), EINVAL), (dict(lddx=47), EINVAL),
    (dict(lddw1=47), EINVAL), (dict(lddw2=39), EINVAL), (dict(db1=P + 2), EINVAL), (dict(dw1=P + 2), EINVAL), (dict(wb=0), EWORKSPACE),
    (dict(ws=None), EINVAL), (dict(ws=P + 128), EINVAL), (dict(dx=None, dw1=None, db1=None, dw2=None, dy=None), OK),
])
def test_gated_bwd_refuses(kw, want):
    assert backward(**kw) == want


def test_gated_workspaces():
    lib = B.load()
    f = lib.mfac_gated_linear_workspace_bytes
    assert f(B.MFAC_BF16, 8192, 2048, 8192, P, 2048, P, 2048) == 0
    assert f(B.MFAC_F32, 8192, 2048, 8192, P, 2048, P, 2048) >= 6 * 2048 * (8192 + 16384)
    assert f(B.MFAC_BF16, 0, 64, 64, P, 64, P, 64) == f(9, 8, 64, 64, P, 64, P, 64) == f(0, 8, 64, 1 << 21, P, 64, P, 64) == 0
    g = lib.mfac_gated_bwd_workspace_bytes

    def need(gtype, wanted, hidden=8192, type=B.MFAC_BF16, rows=8192):
        return g(type, gtype, rows, 2048, hidden, 2048, P, 2048, P, hidden, P, 2048, P, 2048, wanted)

    dz, a, da = 8192 * 16384 * 2, 8192 * 8192 * 2, 8192 * 8192 * 4
    every = B.MFAC_GATED_DX | B.MFAC_GATED_DW1 | B.MFAC_GATED_DW2
    assert need(B.MFAC_BF16, B.MFAC_GATED_DX) == dz                     # dz alone, from the product itself
    assert need(B.MFAC_BF16, every) == dz + a
    assert need(B.MFAC_BF16, B.MFAC_GATED_DW2) == a and need(B.MFAC_BF16, B.MFAC_GATED_DB1) < da + dz
    assert need(B.MFAC_F32, every) == 2 * (dz + a)                      # in two parts
    assert need(B.MFAC_BF16, every | B.MFAC_GATED_DB1) >= dz + a + da   # da is stored where its sums are wanted
    assert need(B.MFAC_F32, every, type=B.MFAC_F32) >= 3 * (dz + a) + da
    assert need(B.MFAC_BF16, 0) == need(B.MFAC_BF16, 32) == need(B.MFAC_F16, every) == 0


def residual(**kw):
    a = dict(type=B.MFAC_BF16, wtype=B.MFAC_F32, norms=POST | PRE, rows=4, cols=64, y=P, ldy=64, post_w=P, post_b=None, gate=P,
             gates=None, ldgates=0, res=P, ldres=64, scale=1.0, p=0.1, at=P, pre_w=P, pre_b=None, eps=1e-6, s=P, lds=64, h=P,
             ldh=64, post_mean=None, post_rstd=P, pre_mean=None, pre_rstd=P, q=None, ldq=0, sq=None)
    a.update(kw)
    return B.mfac_residual_norm(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(type=3), dict(wtype=B.MFAC_F16), dict(norms=8), dict(norms=-1), dict(norms=LAYER), dict(rows=-1), dict(cols=0),
    dict(cols=(1 << 15) + 1, ldy=1 << 16, ldres=1 << 16, lds=1 << 16, ldh=1 << 16), dict(y=None), dict(ldy=63), dict(y=P + 1),
    dict(post_b=P), dict(pre_b=P), dict(post_mean=P), dict(pre_mean=P), dict(gates=P, ldgates=64), dict(gate=None, gates=P, ldgates=63),
    dict(ldres=63), dict(scale=float("inf")), dict(scale=float("nan")), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(at=None),
    dict(at=P + 4), dict(eps=-1.0), dict(eps=float("nan")), dict(lds=63), dict(h=None), dict(ldh=63), dict(post_rstd=P + 2),
    dict(q=P, ldq=64), dict(q=P, ldq=63, sq=P), dict(norms=PRE), dict(norms=PRE, post_w=None), dict(norms=POST), dict(post_w=P + 2),
    dict(norms=POST, pre_w=None, pre_rstd=None), dict(norms=POST, pre_w=None, pre_rstd=None, h=None, q=P, ldq=64, sq=P),
    dict(norms=POST, pre_w=None, pre_rstd=None, h=None, s=None),
])
def test_residual_norm_refuses(kw):
    assert residual(**kw) == EINVAL


def residual_bwd(**kw):
    a = dict(type=B.MFAC_BF16, wtype=B.MFAC_F32, norms=POST | PRE, rows=4, cols=64, ds=P, ldds=64, dh=P, lddh=64, y=P, ldy=64,
             post_mean=None, post_rstd=P, s=P, lds=64, q=None, ldq=0, sq=None, pre_mean=None, pre_rstd=P, post_w=P, post_b=None,
             gate=P, gates=None, ldgates=0, scale=1.0, p=0.1, at=P, pre_w=P, dy=P, lddy=64, dres=P, lddres=64, dgates=None, lddgates=0,
             dpost_w=P, dpost_b=None, dgate=P, dpre_w=P, dpre_b=None, ws=P, wb=BIG)
    a.update(kw)
    return B.mfac_residual_norm_bwd(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(type=5), EINVAL), (dict(wtype=B.MFAC_F16), EINVAL), (dict(norms=LAYER), EINVAL), (dict(cols=(1 << 15) + 1), EINVAL),
    (dict(rows=-1), EINVAL), (dict(ldds=63), EINVAL), (dict(dh=None), EINVAL), (dict(lddh=1), EINVAL), (dict(y=None), EINVAL),
    (dict(ldy=63), EINVAL), (dict(post_rstd=None), EINVAL), (dict(pre_rstd=None), EINVAL), (dict(s=None), EINVAL), (dict(lds=63), EINVAL),
    (dict(q=P, ldq=64, sq=P), EINVAL), (dict(s=None, q=P, ldq=64), EINVAL), (dict(s=None, q=P, ldq=63, sq=P), EINVAL),
    (dict(norms=POST | PRE | LAYER), EINVAL), (dict(norms=POST | PRE | LAYER, post_mean=P), EINVAL), (dict(pre_mean=P), EINVAL),
    (dict(post_b=P), EINVAL), (dict(dpost_b=P), EINVAL), (dict(dpre_b=P), EINVAL), (dict(gates=P, ldgates=64), EINVAL),
    (dict(gate=None), EINVAL), (dict(dgates=P, lddgates=64), EINVAL), (dict(gate=None, dgate=None, gates=P, ldgates=64, dgates=P), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(p=2.0), EINVAL), (dict(at=None), EINVAL), (dict(lddy=63), EINVAL), (dict(lddres=63), EINVAL),
    (dict(norms=PRE), EINVAL), (dict(norms=POST), EINVAL), (dict(dpre_w=P + 2), EINVAL), (dict(wb=8), EWORKSPACE),
    (dict(ws=P + 8), EINVAL), (dict(norms=POST, ds=None, dh=None, s=None, pre_rstd=None, pre_w=None, dpre_w=None), EINVAL),
])
def test_residual_norm_bwd_refuses(kw, want):
    assert residual_bwd(**kw) == want


def test_residual_norm_workspace():
    f = B.load().mfac_residual_norm_bwd_workspace_bytes
    assert f(B.MFAC_BF16, PRE, 16384, 4096) == 512 * 2 * 4096 * 4
    assert f(B.MFAC_BF16, PRE | LAYER, 16384, 4096) == 512 * 4 * 4096 * 4
    assert f(B.MFAC_BF16, PRE, 0, 100) > 0 and f(B.MFAC_BF16, LAYER, 4, 100) == f(4, PRE, 4, 100) == f(B.MFAC_BF16, PRE, 4, 0) == 0


@pytest.mark.parametrize("kw", [dict(type=3), dict(rows=-1), dict(cols=0), dict(x=None), dict(y=None), dict(ldx=63), dict(ldy=63),
                                dict(p=-1.0), dict(p=float("nan")), dict(p=1.5), dict(at=None), dict(at=P + 4), dict(p=0.0, at=None),
                                dict(x=P + 1)])
def test_dropout_refuses(kw):
    a = dict(type=B.MFAC_BF16, rows=4, cols=64, x=P, ldx=64, p=0.5, at=P, y=P, ldy=64)
    a.update(kw)
    assert B.mfac_dropout(*a.values(), None) == EINVAL


def test_no_rows_is_nothing_to_do():
    assert residual(rows=0) == gated(rows=0) == B.mfac_dropout(0, 0, 64, None, 64, 0.5, P, None, 64, None) == OK
    assert backward(rows=0, dw1=None, dw2=None, db1=None, dx=None) == OK


@pytest.mark.parametrize("kw", [dict(type=3), dict(rows=0), dict(cin=0), dict(hidden=0), dict(hidden=(1 << 20) + 1), dict(plan=None),
                                dict(cin=(1 << 21) + 1)])
def test_gated_plan_refuses(kw):
    import ctypes
    a = dict(type=B.MFAC_BF16, hidden_bwd=0, rows=64, cin=64, hidden=64, plan=(ctypes.c_int32 * 3)())
    a.update(kw)
    assert B.mfac_gated_plan(*a.values()) == EINVAL
