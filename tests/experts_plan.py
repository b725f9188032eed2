"""Which kernel a product over groups takes, as the library says it."""
import ctypes
from collections import namedtuple

import torch

from paper_2209_02882_amd import binding

TILES, FEW, REGISTERS = 0, 1, 2
Plan = namedtuple("Plan", "way rows columns wide apart short")
# sizes of groups, K, N: with X beyond 4 GiB these take every tile that such an X is multiplied by
BEYOND_4_GIB = [([200, 0, 360], 136, 4_104), ([3_000, 1, 2_500], 1_032, 4_096), ([512, 300, 0, 700, 1_100, 5, 900, 579], 136, 1_032)]
DTYPES = {torch.float32: binding.SGAP_F32, torch.float16: binding.SGAP_F16, torch.bfloat16: binding.SGAP_BF16}


def plan(G, R, K, N, dtype, layout, gradient=False, ldx=None, x_rows=None, ldy=None, given=True, aligned=True, compute_units=256):
    out = (ctypes.c_int * 6)()
    binding._check(binding.load().sgap_debug_grouped_plan(
        G, R, K, N, DTYPES[dtype], int(given), ldx or K, R if x_rows is None else x_rows, ldy or N, binding.WEIGHT_LAYOUTS[layout],
        int(gradient), int(aligned), compute_units, out))
    return Plan(*out)
