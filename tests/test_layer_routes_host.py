"""Which way the layer's products go, as far as the public size queries tell (no GPU)."""
import pytest

import mx4_ref as ref
from paper_2205_03494_amd import omc


@pytest.mark.parametrize("M,N,K", [(1, 33, 1 << 20), (16, 16, 131072), (32, 33, 1 << 20), (17, 512, 24576), (32, 128, 65536), (16, 2048, 49152)])
def test_a_long_contraction_of_few_rows_is_cut_over_the_chip(M, N, K):
    """33 x 2^20 would keep three of 256 compute units busy for 0.3 - 0.7 ms; parts of a cut one need a workspace."""
    assert omc.omc_mx4_gemm_workspace_bytes(M, N, K) >= 2 * 4 * M * N


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (16, 512, 32768), (32, 8192, 8192), (32, 16, 16384), (1, 8192, 49152), (16, 16384, 65536)])
def test_few_rows_of_shorter_or_wider_ones_need_no_workspace(M, N, K):
    assert omc.omc_mx4_gemm_workspace_bytes(M, N, K) == 0


@pytest.mark.parametrize("M,N,K", [(1, 8192, 2048), (32, 8192, 2048), (20, 8192, 8192), (8192, 20, 30), (8192, 300, 20), (16000, 300, 32), (1 << 20, 33, 32)])
def test_a_product_of_few_rows_and_a_long_contraction_goes_its_own_way(M, N, K):
    """In tiles dX of 1 x 8192 x 2048 takes 14.3 us, 8.1 its own way; all three gradients 29.5 together and 30.5 apart."""
    assert ref.pair_tile(M, N, K) == -1


@pytest.mark.parametrize("M,N,K", [(1, 1024, 4096), (16, 4096, 4096), (20, 300, 300), (1000, 1000, 32), (8192, 4096, 32)])
def test_short_ones_go_together(M, N, K):
    """All three gradients of 16 x 4096 x 4096 take 25.7 us together, 29.0 apart; 8192 x 4096 x 32 37.7 and 50.4."""
    assert ref.pair_tile(M, N, K) > 0


def test_gradients_larger_than_the_caches_in_either_tile():
    from test_gpu_layer_paths import LARGE_GRADIENTS
    assert {ref.pair_tile(*shape) for shape in LARGE_GRADIENTS} == {1, 2} and all(2 * M * K >= 1 << 25 and K % 64 == 0 for M, _, K in LARGE_GRADIENTS)
