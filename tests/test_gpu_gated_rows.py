"""What lies between two blocks over more rows than the card holds at once: the row that is loaded ahead, what one row leaves
for the next, and the last, partly filled turn."""

import pytest
import torch

from gpu_common import require_gpu, say
from test_gpu_gated_ops import rand

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


# more rows than work-groups (their rows, up to 512 columns) in each class of threads a row, of either direction
MANY = [(4501, 40), (2500, 1000), (1100, 2048), (1101, 4093), (700, 8192), (1030, 8200)]


@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_residual_norm_of_many_rows(dev, kind, dtype, rows, cols):
    """Against 64 bits, with every combination of norms, gates and dropout, forward and backward."""
    from test_gpu_gated_ops import test_residual_norm as of_size
    of_size(dev, kind, dtype, rows, cols)


@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("layer", [False, True])
def test_many_rows_in_place(dev, layer, rows, cols):
    """s over y or the residual while the next row is on its way, dy and dresidual over ds and dh."""
    from paper_2107_03356_amd import _binding as B
    from paper_2107_03356_amd import nn
    say("many rows in place", layer, rows, cols)
    kind, norms = ("layer", 7) if layer else ("rms", 3)
    y, r, ds, dh = (rand(dev, s, rows, cols, dtype=BF16) for s in (1, 2, 3, 4))
    w1, w2 = rand(dev, 5, cols, at=1), rand(dev, 6, cols, at=1)
    b1, b2 = (rand(dev, s, cols) if layer else None for s in (7, 8))
    ptr = lambda t: None if t is None else t.data_ptr()   # noqa: E731
    o = nn.residual_norm_forward(y, r, post=(w1, b1), pre=(w2, b2), kind=kind)
    g = nn.residual_norm_backward(ds, dh, y, o.s, o.post, o.pre, post=(w1, b1), pre=(w2, b2), kind=kind)
    st = torch.cuda.current_stream().cuda_stream
    for s_at in (0, 1):
        t, h = [y.clone(), r.clone()], torch.empty_like(y)
        assert B.mfac_residual_norm(
            B.MFAC_BF16, B.MFAC_F32, norms, rows, cols, ptr(t[0]), cols, ptr(w1), ptr(b1), None, None, 0, ptr(t[1]), cols, 1.0, 0.0,
            None, ptr(w2), ptr(b2), 1e-6, ptr(t[s_at]), cols, ptr(h), cols, None, None, None, None, None, 0, None, st) == B.MFAC_OK
        assert torch.equal(t[s_at], o.s) and torch.equal(h, o.h)
    a, b = ds.clone(), dh.clone()
    assert B.mfac_residual_norm_bwd(
        B.MFAC_BF16, B.MFAC_F32, norms, rows, cols, ptr(a), cols, ptr(b), cols, ptr(y), cols, ptr(o.post[0]), ptr(o.post[1]), ptr(o.s),
        cols, None, 0, None, ptr(o.pre[0]), ptr(o.pre[1]), ptr(w1), ptr(b1), None, None, 0, 1.0, 0.0, None, ptr(w2), ptr(b), cols,
        ptr(a), cols, None, 0, None, None, None, None, None, None, 0, st) == B.MFAC_OK
    assert torch.equal(b, g.dy) and torch.equal(a, g.dresidual)
