"""Sizes at the ends of what the calls of a mixture of experts take: refused on the host where 32-bit positions would not
hold what a kernel counts.  No GPU."""
import pytest

from paper_2209_02882_amd import binding
from test_experts_refusals import COMBINE, COMBINE_GRAD, GRAD, MM, ROUTE, W4, WGRAD, refused

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


# sizes whose products pass 64 bits, and would come back as small ones
@pytest.mark.parametrize("T,k", [(2**62, 4), (2**60, 16), (2**63 - 1, 2), (2**61 + 1, 8)])
def test_numbers_of_pairs_beyond_64_bits(T, k):
    with pytest.raises(binding.SgapError, match="int32"):
        binding.sgap_route_topk_workspace_size(T, 16, k)
    refused("sgap_route_topk", ROUTE, "int32", T=T, k=k, bytes=2**62)
    refused("sgap_route_topk_grad", GRAD, "int32", T=T, k=k)
    refused("sgap_route_combine", COMBINE, "int32", T=T, k=k)
    refused("sgap_route_combine_grad", COMBINE_GRAD, "int32", T=T, k=k)


@pytest.mark.parametrize("G,K,N", [(2**20, 2**30, 2**30), (2**16, 2**30, 2**25), (2**20, 2**26, 2**24), (2**12, 2**31 - 65536, 2**31 - 65536)])
def test_4_bit_weights_beyond_64_bits(G, K, N):
    for zeros in (0, 1):
        assert binding.load().sgap_w4_layout_size(G, K, N, 32, zeros) == -1
    refused("sgap_grouped_mm_w4", W4, "memory", G=G, K=K, N=N, ldx=K, ldy=N, group_k=32)
    args = dict(G=G, K=K, N=N, group_k=32, codes=16, scales=16, zeros=16, weights=16, bytes=2**62, stream=None)
    refused("sgap_w4_layout", args, "memory")


def test_the_largest_4_bit_weights_have_their_size():
    # 2^20 groups of 2^12 x 2^12: 8 TB of codes, a scale of two bytes for each 32
    assert binding.sgap_w4_layout_size(2**20, 2**12, 2**12, 32) == 2**43 + 2**44 // 32 * 2
