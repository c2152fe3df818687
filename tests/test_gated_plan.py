"""What a gated layer's products are said to run: their stores past the caches, by what is kept (no GPU needed)."""

import ctypes
import os

import pytest

from paper_2107_03356_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmfac.so not built")


def plan(product, rows, cin, hidden, dtype=B.MFAC_BF16):
    p = (ctypes.c_int32 * 3)()
    assert B.mfac_gated_plan(dtype, product, rows, cin, hidden, p) == B.MFAC_OK
    return tuple(p)


@pytest.mark.parametrize("product,rows,cin,hidden,want", [
    # 256 MB are the last-level cache. x, W and y: 235 million bytes; the pre-activations are 268 million more, copies 134
    (B.MFAC_GATED_FORWARD, 8192, 2048, 8192, (256, 1, 0)),
    (B.MFAC_GATED_FORWARD_Z, 8192, 2048, 8192, (256, 1, 1)),
    (B.MFAC_GATED_FORWARD_COPIES, 8192, 2048, 8192, (256, 1, 1)),
    (B.MFAC_GATED_FORWARD_COPIES, 2048, 2048, 8192, (256, 1, 0)),
    (B.MFAC_GATED_FORWARD, 16384, 2048, 8192, (256, 1, 1)),
    # dz from the product's own epilogue is never stored past the caches; da in fp32, 537 million bytes, is
    (B.MFAC_GATED_HIDDEN, 16384, 2048, 8192, (256, 1, 0)),
    (B.MFAC_GATED_HIDDEN_SUMS, 16384, 2048, 8192, (256, 1, 1)),
    (B.MFAC_GATED_HIDDEN, 16384, 2048, 8200, (256, 1, 1)),
    (B.MFAC_GATED_HIDDEN, 8192, 512, 4104, (256, 1, 0)),
])
def test_gated_plan_is_what_runs(product, rows, cin, hidden, want):
    assert plan(product, rows, cin, hidden) == want


def test_gated_plan_refuses_what_it_does_not_know():
    p = (ctypes.c_int32 * 3)()
    for product in (-1, 5):
        assert B.mfac_gated_plan(B.MFAC_BF16, product, 64, 64, 64, p) == B.MFAC_EINVAL
