"""Which kernel a product over groups takes, as the library says it."""
import ctypes
from collections import namedtuple

import torch

from paper_2209_02882_amd import binding

TILES, FEW, REGISTERS = 0, 1, 2
Plan = namedtuple("Plan", "way rows columns wide apart short")
DTYPES = {torch.float32: binding.SGAP_F32, torch.float16: binding.SGAP_F16, torch.bfloat16: binding.SGAP_BF16}


def plan(G, R, K, N, dtype, layout, gradient=False, ldx=None, x_rows=None, ldy=None, given=True, aligned=True, compute_units=256):
    out = (ctypes.c_int * 6)()
    binding._check(binding.load().sgap_debug_grouped_plan(
        G, R, K, N, DTYPES[dtype], int(given), ldx or K, R if x_rows is None else x_rows, ldy or N, binding.WEIGHT_LAYOUTS[layout],
        int(gradient), int(aligned), compute_units, out))
    return Plan(*out)
