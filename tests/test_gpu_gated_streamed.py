"""Gated layers whose results are stored past the caches, against 64 bits."""

import pytest
import torch

from gated_cases import gated_plan
from gated_ref import gate_slopes64, gated64, rounded
from gpu_common import require_gpu, say
from paper_2107_03356_amd import _binding as B
from test_gpu_gated_ops import copy_holds, forward_reference, halves, holds, rand
from train_ref import E32, TINY, growth

pytestmark = pytest.mark.gpu

CODES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}


@pytest.fixture(scope="module")
def dev():
    return require_gpu()


@pytest.mark.parametrize("hid", [16384, 16403])
@pytest.mark.parametrize("dtype", list(CODES))
def test_gated_forward_past_the_caches(dev, dtype, hid):
    """Tiles of 256 that are stored with nontemporal stores, whole and with edges in both directions; with nothing, the
    pre-activations or their copies kept."""
    from paper_2107_03356_amd import nn
    say("gated forward past the caches", dtype, hid)
    rows, cin = 8229, 72
    for product in (B.MFAC_GATED_FORWARD, B.MFAC_GATED_FORWARD_Z, B.MFAC_GATED_FORWARD_COPIES):
        assert gated_plan(CODES[dtype], product, rows, cin, hid) == (256, 1, 1)
    x, w, b = rand(dev, 1, rows, cin, dtype=dtype), rand(dev, 2, 2 * hid, cin, dtype=dtype, scale=cin ** -0.5), rand(dev, 3, 2 * hid)
    z, e = forward_reference(x, w, b)
    y64, ye = gated64("silu", *z, *e)
    y = nn.gated_linear_forward(x, w, b)
    holds(y, y64, rounded(y64, ye, dtype, TINY[dtype]), "y")
    del y64, ye
    yz, kept = nn.gated_linear_forward(x, w, b, keep="z")
    for i in range(2):
        holds(kept[i], z[i], rounded(z[i], e[i], dtype, TINY[dtype]), "z")
    del kept
    y8, copies = nn.gated_linear_forward(x, w, b, keep="pack8")
    assert torch.equal(yz, y) and torch.equal(y8, y)
    for i in range(2):
        copy_holds(copies[i], z[i], e[i], "copy")


def test_stored_da_past_the_caches(dev):
    """Where db is wanted, da goes through memory in fp32. The identity as a half of w1 shows dz."""
    from paper_2107_03356_amd import nn
    say("stored da past the caches")
    dtype, rows, dim, hid = torch.bfloat16, 16413, 72, 4200
    assert gated_plan("bf16", B.MFAC_GATED_HIDDEN_SUMS, rows, dim, hid) == (256, 1, 1)
    dy, w2 = rand(dev, 1, rows, dim, dtype=dtype), rand(dev, 2, dim, hid, dtype=dtype, scale=dim ** -0.5)
    z = rand(dev, 3, rows, hid, dtype=dtype), rand(dev, 4, rows, hid, dtype=dtype)
    da, ed = dy.double() @ w2.double(), E32 * growth(dim) * (dy.double().abs() @ w2.double().abs())
    slopes = gate_slopes64("silu", z[0].double(), z[1].double(), da, ed)[:2]
    del da, ed
    for i, (w1, (v, e)) in enumerate(zip(halves(dev, hid, dtype), slopes)):
        dx, _, db, _, _ = nn.gated_feed_forward_backward(dy, None, w1, w2, z, need=(True, False, True, False, False))
        holds(dx, v, rounded(v, e, dtype, TINY[dtype]), "dz")
        holds(db[i * hid:(i + 1) * hid], v.sum(0), E32 * (rows / 4 + 60) * v.abs().sum(0) + e.sum(0), "db")
