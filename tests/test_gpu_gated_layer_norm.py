"""A layer norm with nothing else between two blocks is layer_norm, forward and backward."""

import pytest
import torch

from gpu_common import require_gpu, say
from test_gpu_gated_ops import rand
from train_ref import U

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (100, 40), (2100, 512), (33, 1000), (300, 2047), (130, 4096), (40, 9000),
                                       (5, 16391), (2, 32768)])
@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16)])
def test_layer_norm_alone(dev, dtype, wt, rows, cols):
    from paper_2107_03356_amd import nn
    say("layer norm alone", dtype, wt, rows, cols)
    x, dh, ds = (rand(dev, s, rows, cols, dtype=dtype, pad=cols % 3) for s in (1, 2, 3))
    w, b = rand(dev, 4, cols, dtype=wt, at=1, scale=0.2), rand(dev, 5, cols, dtype=wt)
    for norm in ((w, b), (w, None), (None, None)):
        y, mean, rstd = nn.layer_norm_forward(x, *norm, eps=1e-5)
        yp, copy, _ = nn.layer_norm_forward(x, *norm, eps=1e-5, pack=True)
        o = nn.residual_norm_forward(x, pre=norm, kind="layer", eps=1e-5, pack=True)
        assert torch.equal(o.h, y) and torch.equal(o.h, yp) and torch.equal(o.copy.q, copy.q) and torch.equal(o.copy.s, copy.s)
        assert torch.equal(o.pre[0], mean) and torch.equal(o.pre[1], rstd)
        for add in (ds, None):
            for kept in (x, copy):
                m = mean if kept is x else None
                dx, dw, db = nn.layer_norm_backward(dh, kept, m, rstd, norm[0], add=add)
                g = nn.residual_norm_backward(add, dh, None, kept, None, (m, rstd), pre=norm, kind="layer")
                assert torch.equal(g.dy, dx) and g.dresidual is g.dy
                assert norm[0] is None or torch.equal(g.dpre[0], dw)
                assert norm[1] is None or torch.equal(g.dpre[1], db)
                # a scaled residual has a gradient of its own, and another kernel: both round to dtype (U of it each), and
                # rstd, 316 at most, brings a few units of fp32's sums of dh, which is below 8, to 316 * 8 * 32 * 2^-24
                half = nn.residual_norm_backward(add, dh, None, kept, None, (m, rstd), pre=norm, kind="layer", scale=0.5)
                torch.testing.assert_close(half.dy.double(), dx.double(), rtol=2 * U[dtype], atol=5e-3 + 2 * U[dtype])


def test_layer_norm_alone_in_place_and_without_dx(dev):
    """h over y, dy over ds or dh, as the header allows; the parameters' gradients without dy."""
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("layer norm alone in place")
    st = torch.cuda.current_stream().cuda_stream
    for rows, cols in ((300, 100), (40, 9000), (6, 20000)):
        x, ds, dh = (rand(dev, s, rows, cols, dtype=BF16) for s in (1, 2, 3))
        w, b = rand(dev, 4, cols, at=1), rand(dev, 5, cols)
        o = nn.residual_norm_forward(x, pre=(w, b), kind="layer")
        g = nn.residual_norm_backward(ds, dh, None, x, None, o.pre, pre=(w, b), kind="layer")
        t = x.clone()
        assert B.mfac_residual_norm(B.MFAC_BF16, B.MFAC_F32, 6, rows, cols, t.data_ptr(), cols, None, None, None, None, 0, None, 0, 1.0,
                                    0.0, None, w.data_ptr(), b.data_ptr(), 1e-6, None, 0, t.data_ptr(), cols, None, None, None, None,
                                    None, 0, None, st) == B.MFAC_OK
        assert torch.equal(t, o.h)
        need = B.mfac_residual_norm_bwd_workspace_bytes(B.MFAC_BF16, 6, rows, cols)
        ws, grads = torch.empty(need, dtype=torch.uint8, device=dev), torch.empty(2, cols, device=dev)
        for at in ("ds", "dh", None):
            t = {"ds": ds.clone(), "dh": dh.clone()}
            assert B.mfac_residual_norm_bwd(
                B.MFAC_BF16, B.MFAC_F32, 6, rows, cols, t["ds"].data_ptr(), cols, t["dh"].data_ptr(), cols, None, 0, None, None,
                x.data_ptr(), cols, None, 0, None, o.pre[0].data_ptr(), o.pre[1].data_ptr(), None, None, None, None, 0, 1.0, 0.0, None,
                w.data_ptr(), t[at].data_ptr() if at else None, cols, None, 0, None, 0, None, None, None, grads[0].data_ptr(),
                grads[1].data_ptr(), ws.data_ptr(), need, st) == B.MFAC_OK
            if at:
                assert torch.equal(t[at], g.dy) and torch.equal(grads[0], g.dpre[0]) and torch.equal(grads[1], g.dpre[1])
            else:
                torch.testing.assert_close(grads[0], g.dpre[0], rtol=1e-4, atol=1e-3)
                torch.testing.assert_close(grads[1], g.dpre[1], rtol=1e-4, atol=1e-3)
