"""Which kernel a linear layer's products take (no GPU needed): the sizes that the GPU tests hold each kernel to its definition at."""

import ctypes
import os

import pytest

from paper_2107_03356_amd import _binding as B
from train_cases import PRODUCTS, layer, plan, runs

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmfac.so not built")


@pytest.mark.parametrize("product", [B.MFAC_PRODUCT_FORWARD, B.MFAC_PRODUCT_INPUT, B.MFAC_PRODUCT_WEIGHT])
@pytest.mark.parametrize("size,want,types", PRODUCTS)
def test_sizes_take_the_kernel_that_they_are_for(product, size, want, types):
    for t in types:
        for o in {t, "f32"} if product == B.MFAC_PRODUCT_WEIGHT else {t}:
            assert runs(t, o, product, size, want), (t, o, plan(t, o, product, *layer(product, *size)))


def test_few_rows_take_the_kernel_for_them():
    for t in ("f32", "bf16", "f16"):
        assert plan(t, t, B.MFAC_PRODUCT_FORWARD, 16, 4096, 4096) == (0, 1, 0)
        assert plan(t, t, B.MFAC_PRODUCT_FORWARD, 17, 4096, 4096)[0] > 0
        assert plan(t, t, B.MFAC_PRODUCT_INPUT, 1, 4096, 4096)[0] > 0


def test_plan_and_workspace_agree():
    """Operands that are taken as they are need room for parts only."""
    for rows, cin, cout in ((3000, 520, 3080), (304, 4104, 520), (1104, 4104, 1032)):
        _, parts, _ = plan("bf16", "bf16", B.MFAC_PRODUCT_FORWARD, rows, cin, cout)
        need = B.mfac_linear_workspace_bytes(B.MFAC_BF16, rows, cin, cout, 1 << 20, cin, 1 << 20, cin)
        assert need == (0 if parts == 1 else -(-rows * cout * parts * 4 // 256) * 256)


@pytest.mark.parametrize("kw", [dict(type=3), dict(type=-1), dict(otype=B.MFAC_F16), dict(product=3), dict(product=-1),
                                dict(rows=0), dict(rows=(1 << 30) + 1), dict(cin=0), dict(cout=0), dict(cin=(1 << 21) + 1),
                                dict(cout=(1 << 21) + 1), dict(packed=1), dict(plan=None)])
def test_plan_refuses(kw):
    a = dict(type=B.MFAC_BF16, otype=B.MFAC_BF16, product=B.MFAC_PRODUCT_FORWARD, rows=8, cin=64, cout=64, packed=0,
             plan=(ctypes.c_int32 * 3)())
    a.update(kw)
    assert B.mfac_linear_plan(*a.values()) == B.MFAC_EINVAL
