"""Sizes by which a linear layer's three products run each kernel, and how to ask the library which one it takes."""

import ctypes

from paper_2107_03356_amd import _binding as B

# (M, N, K) of C (M x N) = A B^T, with the tile, the parts of K and whether C is stored past the caches that it is there
# for, in the types given. M and N are odd where a tile's edge is to fall inside a store's eight columns.
PRODUCTS = [
    ((3001, 3077, 520), (256, 1, 0), ("bf16", "f16", "f32")),
    ((4099, 8197, 8200), (256, 1, 1), ("bf16", "f16", "f32")),
    ((2051, 2053, 200), (128, 1, 0), ("bf16", "f16", "f32")),
    ((1003, 1045, 264), (64, 1, 0), ("bf16", "f16", "f32")),
    ((2050, 2056, 1032), (256, 3, 0), ("f32",)),
    ((1101, 1029, 4104), (128, 6, 0), ("bf16", "f16", "f32")),
    ((301, 523, 4104), (64, None, 0), ("bf16", "f16", "f32")),
]
CODES = {"f32": B.MFAC_F32, "bf16": B.MFAC_BF16, "f16": B.MFAC_F16}


def layer(product, M, N, K):
    """(rows, cin, cout) of the layer whose forward, input or weight product has these sizes."""
    return {B.MFAC_PRODUCT_FORWARD: (M, K, N), B.MFAC_PRODUCT_INPUT: (M, N, K), B.MFAC_PRODUCT_WEIGHT: (K, N, M)}[product]


def plan(dtype, otype, product, rows, cin, cout, packed=False):
    """(tile, parts, streams)"""
    p = (ctypes.c_int32 * 3)()
    assert B.mfac_linear_plan(CODES[dtype], CODES[otype], product, rows, cin, cout, int(packed), p) == B.MFAC_OK
    return tuple(p)


def runs(dtype, otype, product, size, want, packed=False):
    """Whether the product of these sizes takes the kernel that `want` names (parts None: two or more)."""
    tile, parts, streams = plan(dtype, otype, product, *layer(product, *size), packed)
    return tile == want[0] and (parts > 1 if want[1] is None else parts == want[1]) and streams == want[2]
