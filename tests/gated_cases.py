"""How to ask the library which kernel a gated layer's product takes."""

import ctypes

from paper_2107_03356_amd import _binding as B
from train_cases import CODES


def gated_plan(dtype, hidden_bwd, rows, cin, hidden):
    """(tile, parts, streams) of the layer's product, or of that behind it in the backward pass (cin is its cout)."""
    p = (ctypes.c_int32 * 3)()
    assert B.mfac_gated_plan(CODES[dtype], int(hidden_bwd), rows, cin, hidden, p) == B.MFAC_OK
    return tuple(p)
