"""Which kernel a product of numbers of 8 bits takes.  No GPU."""
import ctypes

import pytest
import torch

from experts_plan import DTYPES
from paper_2209_02882_amd import binding

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def plan(G, R, K, N, dtype, given=True, src=False, x_rows=None, compute_units=256):
    out = (ctypes.c_int * 4)()
    binding._check(binding.load().sgap_debug_f8_plan(G, R, K, N, DTYPES[dtype], int(given), int(src), R if x_rows is None else x_rows,
                                                     compute_units, out))
    return tuple(out)


@pytest.mark.parametrize("G,R,K,N,dtype,want", [
    (1, 1, 4_096, 4_096, BF16, (0, 16, 16, 0)),
    (1, 32, 8_192, 8_192, BF16, (0, 32, 32, 0)),
    (8, 8, 8_192, 1_024, F16, (0, 16, 16, 0)),
    (64, 64, 2_048, 1_408, F16, (0, 16, 16, 2)),
    (1, 128, 4_096, 256, BF16, (0, 16, 16, 0)),
    (1, 256, 4_096, 4_096, BF16, (2, 64, 128, 0)),
    (1, 1_024, 4_096, 4_096, BF16, (2, 128, 128, 0)),
    (1, 2_048, 4_096, 4_096, BF16, (1, 128, 128, 0)),
    (1, 256, 512, 4_096, BF16, (1, 64, 128, 0)),            # blocks too few to share
    (1, 8_192, 4_096, 8_192, BF16, (1, 256, 256, 0)),
    (16, 16_384, 2_048, 4_096, BF16, (1, 256, 256, 0)),
    (1, 8_192, 4_096, 8_192, F32, (1, 128, 128, 0)),
    (8, 4_096, 1_024, 1_024, F32, (1, 64, 128, 0)),
    (7, 3_001, 1_000, 1_531, F16, (1, 64, 128, 0)),
    (4, 4_000, 0, 500, BF16, (0, 32, 32, 0)),              # nothing to multiply
    (1, 4_096, 1 << 23, 512, BF16, (0, 32, 32, 0)),        # columns' codes 8 MiB apart
])
def test_products(G, R, K, N, dtype, want):
    assert plan(G, R, K, N, dtype) == want


def test_rows_gathered_from_more_than_4_gib():
    assert plan(1, 16_384, 4_096, 4_096, BF16, src=True, x_rows=1 << 20)[3] == 0
    assert plan(1, 16_384, 4_096, 4_096, BF16, src=True, x_rows=(1 << 20) + 1) == (1, 128, 128, 1)
    assert plan(1, 16_384, 4_096, 4_096, BF16, x_rows=1 << 22) == (1, 256, 256, 0)


def test_bad_arguments():
    for bad in (dict(G=0), dict(R=-1), dict(N=2**31 - 1), dict(compute_units=0), dict(x_rows=-1)):
        with pytest.raises(binding.SgapError):
            plan(**{**dict(G=1, R=1, K=1, N=1, dtype=BF16), **bad})
