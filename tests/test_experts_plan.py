"""Which kernel a product over groups takes.  No GPU."""
import ctypes

import pytest
import torch

from experts_plan import BEYOND_4_GIB, DTYPES, FEW, REGISTERS, TILES, plan
from paper_2209_02882_amd import binding

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("G,R,K,N,dtype,layout,want", [
    (16, 16_384, 2_048, 4_096, BF16, "nk", (TILES, 256, 256, 0, 0, 0)),
    (64, 8_192, 1_024, 2_048, BF16, "nk", (TILES, 128, 128, 0, 0, 0)),
    (16, 32, 2_048, 4_096, BF16, "nk", (TILES, 64, 128, 0, 1, 0)),    # every weight passes once: rows of 4,096 bytes
    (16, 32, 2_040, 4_096, BF16, "nk", (TILES, 64, 128, 0, 0, 0)),
    (16, 32, 2_048, 4_096, BF16, "kn", (TILES, 64, 128, 0, 0, 0)),
    (8, 4_096, 1_024, 1_024, F32, "nk", (TILES, 64, 128, 0, 0, 0)),
    (1, 1, 4_096, 4_096, BF16, "nk", (FEW, 16, 16, 0, 0, 0)),
    (1, 1, 4_096, 4_096, BF16, "kn", (FEW, 16, 32, 0, 0, 0)),
    (8, 8, 64, 4_096, F16, "nk", (FEW, 16, 32, 0, 0, 0)),
    (1, 512, 4_096, 512, BF16, "nk", (FEW, 32, 32, 0, 0, 0)),
    (1, 128, 4_096, 4_096, BF16, "kn", (FEW, 32, 64, 0, 0, 0)),
    (7, 3_001, 1_000, 1_531, F16, "kn", (REGISTERS, 64, 128, 0, 0, 0)),
    (7, 3_001, 5, 1_531, F16, "kn", (REGISTERS, 32, 128, 0, 0, 1)),
    (100, 3_001, 1_000, 1_531, F16, "kn", (REGISTERS, 32, 128, 0, 0, 0)),
    (7, 30_001, 1_000, 1_531, F16, "kn", (REGISTERS, 128, 128, 0, 0, 0)),
])
def test_products(G, R, K, N, dtype, layout, want):
    assert plan(G, R, K, N, dtype, layout) == want


@pytest.mark.parametrize("G,R,K,N,dtype,want", [
    (16, 16_384, 2_048, 4_096, BF16, (TILES, 256, 256, 0, 0, 0)),
    (8, 4_096, 1_024, 1_024, F32, (TILES, 128, 128, 0, 0, 0)),
    (1, 8_192, 256, 256, BF16, (FEW, 32, 32, 0, 0, 0)),
    (1, 8_192, 1_024, 1_024, BF16, (FEW, 64, 64, 0, 0, 0)),
    (7, 3_001, 1_000, 1_531, F16, (REGISTERS, 128, 128, 0, 0, 0)),
    (7, 3_001, 1_000, 7, F16, (REGISTERS, 128, 128, 0, 0, 1)),
])
def test_gradients_of_weights(G, R, K, N, dtype, want):
    for layout in ("nk", "kn"):
        assert plan(G, R, K, N, dtype, layout, gradient=True) == want


def test_what_the_rows_of_x_decide():
    big = dict(G=16, R=16_384, K=2_048, N=4_096, layout="nk")
    for dtype, rows in ((BF16, 2**20), (F32, 2**19)):
        assert not plan(**big, dtype=dtype, x_rows=rows - 1).wide and plan(**big, dtype=dtype, x_rows=rows).wide
        assert plan(**big, dtype=dtype, x_rows=rows, gradient=True).wide
    assert plan(**big, dtype=BF16, ldx=2_052).way == REGISTERS and plan(**big, dtype=F32, ldx=2_052).way == TILES
    assert plan(**big, dtype=BF16, ldy=4_097).way == REGISTERS and plan(**big, dtype=BF16, aligned=False).way == REGISTERS
    assert plan(**big, dtype=BF16, x_rows=0).short


def test_bad_arguments():
    out = (ctypes.c_int * 6)()
    args = dict(G=1, R=4, K=8, N=8, dtype=0, given=1, ldx=8, x_rows=4, ldy=8, layout=0, gradient=0, aligned=1, units=256, plan=out)
    ask = binding.load().sgap_debug_grouped_plan
    assert ask(*args.values()) == 0
    for change in (dict(G=0), dict(R=-1), dict(dtype=3), dict(ldx=7), dict(ldy=7), dict(layout=2), dict(units=0), dict(plan=None),
                   dict(K=2**31 - 1, ldx=2**31)):
        assert ask(*{**args, **change}.values()) == binding.SGAP_ERR_INVALID_ARG


def test_sizes_that_take_every_tile_beyond_4_gib():
    seen = set()
    for sizes, K, N in BEYOND_4_GIB:
        for dtype in DTYPES:
            for layout in ("nk", "kn"):
                for gradient in (False, True):
                    p = plan(len(sizes), sum(sizes), K, N, dtype, layout, gradient, ldx=2**16 + 8, x_rows=36_000)
                    if p.way == TILES:
                        assert p.wide
                        seen.add((dtype, layout, gradient, p.rows))
    want = {(dtype, layout, False, rows) for dtype in DTYPES for layout in ("nk", "kn") for rows in (64, 128)}
    want |= {(dtype, layout, True, 128) for dtype in DTYPES for layout in ("nk", "kn")}
    want |= {(dtype, layout, gradient, 256) for dtype in (F16, BF16) for layout in ("nk", "kn") for gradient in (False, True)}
    assert seen == want
