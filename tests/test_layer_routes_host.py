"""Which way the layer's products go, as far as the public size queries tell (no GPU)."""
import pytest

from paper_2205_03494_amd import omc


@pytest.mark.parametrize("M,N,K", [(1, 33, 1 << 20), (16, 16, 131072), (32, 33, 1 << 20), (17, 512, 24576), (32, 128, 65536), (16, 2048, 49152)])
def test_a_long_contraction_of_few_rows_is_cut_over_the_chip(M, N, K):
    """33 x 2^20 would keep three of 256 compute units busy for 0.3 - 0.7 ms; parts of a cut one need a workspace."""
    assert omc.omc_mx4_gemm_workspace_bytes(M, N, K) >= 2 * 4 * M * N


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (16, 512, 32768), (32, 8192, 8192), (32, 16, 16384), (1, 8192, 49152), (16, 16384, 65536)])
def test_few_rows_of_shorter_or_wider_ones_need_no_workspace(M, N, K):
    assert omc.omc_mx4_gemm_workspace_bytes(M, N, K) == 0
