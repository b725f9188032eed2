"""Sizes at the ends of what the calls of a mixture of experts take: refused on the host where 32-bit positions would not
hold what a kernel counts.  No GPU."""
import pytest

from paper_2209_02882_amd import binding
from test_experts_refusals import MM, W4, WGRAD, refused

MOST = 2**31 - 65536  # room for the kernels' 32-bit positions to pass the end by some tiles


@pytest.mark.parametrize("over", [1, 64, 65534])
@pytest.mark.parametrize("name,args", [("sgap_grouped_mm", MM), ("sgap_grouped_mm_wgrad", WGRAD), ("sgap_grouped_mm_w4", W4)])
def test_rows_and_columns_within_a_tile_of_32_bits(name, args, over):
    big = MOST + over
    refused(name, args, "int32", R=big, x_rows=big)
    refused(name, args, "int32", N=big, ldy=big)


@pytest.mark.parametrize("over", [1, 64, 65534])
@pytest.mark.parametrize("name,args", [("sgap_grouped_mm", MM), ("sgap_grouped_mm_wgrad", WGRAD)])
def test_inner_values_within_a_tile_of_32_bits(name, args, over):
    refused(name, args, "int32", K=MOST + over, ldx=MOST + over)


def test_4_bit_weights_within_a_tile_of_32_bits():
    for K in (MOST + 128, MOST + 65408):
        refused("sgap_grouped_mm_w4", W4, "int32", K=K, ldx=K)
        with pytest.raises(binding.SgapError, match="int32"):
            binding.sgap_w4_layout_size(1, K, 16, 64)
    assert binding.sgap_w4_layout_size(1, MOST, 1, 128) > 0


@pytest.mark.parametrize("name,args", [("sgap_grouped_mm", MM), ("sgap_grouped_mm_wgrad", WGRAD)])
def test_the_largest_sizes_are_not_refused(name, args):
    # found in order: the sizes are looked at before the addresses, and these calls have none
    refused(name, args, "null", R=MOST, x_rows=MOST, Y=None)
    refused(name, args, "null", N=MOST, ldy=MOST, Y=None)
    refused(name, args, "null", K=MOST, ldx=MOST, X=None)
