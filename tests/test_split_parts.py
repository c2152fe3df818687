"""What six of the nine products of two fp32 values' bf16 parts leave out, as the kernels' comments and mfac.h say."""

import numpy as np


def bf16(x):
    """Rounded to bf16, ties to even."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + (u >> 16 & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def parts(x):
    hi = bf16(x)
    mid = bf16(x - hi)
    lo = (x - hi) - mid
    assert np.array_equal(bf16(lo), lo)   # three parts are the value
    return [p.astype(np.float64) for p in (hi, mid, lo)]


def test_three_products_left_out_are_one_fp32_rounding_at_most():
    rng = np.random.default_rng(0)
    x = (1 + rng.integers(0, 1 << 23, 1 << 21) / (1 << 23)).astype(np.float32)
    x[0] = 1.0038986
    hi, mid, lo = parts(x)
    assert np.array_equal(hi + mid + lo, x.astype(np.float64))
    assert np.abs(mid).max() <= 2.0 ** -8 and np.abs(lo).max() <= 2.0 ** -17
    worst = np.argsort(-(np.abs(mid) * 2 ** 8 + np.abs(lo) * 2 ** 17) / x)[:1500]
    h, m, l, v = hi[worst], mid[worst], lo[worst], x[worst].astype(np.float64)
    left = np.abs(np.outer(m, l) + np.outer(l, m) + np.outer(l, l)) / np.outer(v, v)
    assert 2.0 ** -24.1 < left.max() <= 2.0 ** -24 * (1 + 2.0 ** -10)
