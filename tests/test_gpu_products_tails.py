"""Gates far out: their values and slopes by their own magnitude, in the kernel of few rows and in tiles, plain sums and 8-bit ones.  Weights are zero, so that g is its bias and u is one."""
import pytest
import torch

import tails_ref as tails
from paper_2205_03494_amd import omc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GATES = (omc.OMC_GATE_SIGMOID, omc.OMC_GATE_SWISH, omc.OMC_GATE_GELU)


def space(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("h_type", [F32, BF16])
@pytest.mark.parametrize("M", [1, 17, 40, 300])
def test_gated_linear(M, h_type, gate):
    g = tails.arguments(gate, "cuda")
    N, K = g.numel(), 64
    X, W, one = torch.ones(M, K, dtype=BF16, device="cuda"), torch.zeros(N, K, dtype=BF16, device="cuda"), torch.ones(N, device="cuda")
    H, sg, su = torch.zeros(M, N, dtype=h_type, device="cuda"), torch.zeros(M, N, dtype=BF16, device="cuda"), torch.zeros(M, N, dtype=BF16, device="cuda")
    omc.omc_gated_linear(X, W, W, g, one, gate, H, sg, su, space(omc.omc_gated_linear_workspace_bytes(M, N, K)))
    for m in {0, M // 2, M - 1}:
        tails.check(g, H[m], sg[m], su[m], gate)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("h_type", [F32, BF16])
@pytest.mark.parametrize("M", [1, 17, 40, 300])
def test_i8_gated_linear(M, h_type, gate):
    g = tails.arguments(gate, "cuda")
    N, K = g.numel(), 64
    X, one = torch.ones(M, K, dtype=BF16, device="cuda"), torch.ones(N, device="cuda")
    codes = torch.zeros(N, omc.omc_i8_code_bytes(1, K), dtype=torch.uint8, device="cuda")
    H = torch.zeros(M, N, dtype=h_type, device="cuda")
    omc.omc_i8_gated_linear(X, codes, one, codes, one, g, one, gate, H, space(omc.omc_i8_gated_linear_workspace_bytes(M, N, K)))
    for m in {0, M // 2, M - 1}:
        tails.check(g, H[m], None, None, gate)
