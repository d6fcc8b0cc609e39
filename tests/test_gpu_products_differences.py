"""The gated layer's gradients against differences of its own forward pass: few rows and tiles, whole and ragged."""
import pytest
import torch

import differences_ref as differences
from paper_2205_03494_amd import omc

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GATES = (omc.OMC_GATE_SIGMOID, omc.OMC_GATE_SWISH, omc.OMC_GATE_GELU)
SIZES = [(1, 16, 64), (3, 17, 7), (7, 24, 40), (40, 136, 72), (96, 72, 64), (300, 40, 24)]


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("size", SIZES)
def test_gradients_against_differences_that_do_not_cancel(size, gate):
    M, N, K = size
    layer = differences.Layer(M, N, K, gate, 30, "cuda")
    ws = torch.empty(max(16, omc.omc_gated_linear_workspace_bytes(M, N, K), omc.omc_gated_linear_backward_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")

    def objective(X, Wg, Wu, bg, bu, sg=None, su=None):
        H = torch.empty(M, N, device="cuda")
        omc.omc_gated_linear(X, Wg, Wu, bg, bu, gate, H, sg, su, ws)
        return (H.double() * layer.R.double()).sum().item()
    X, Wg, Wu, bg, bu = (layer.at[n] for n in differences.NAMES)
    sg, su = torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")
    objective(X, Wg, Wu, bg, bu, sg, su)
    gradients = {"X": torch.empty(M, K, device="cuda"), "Wg": torch.empty(N, K, device="cuda"), "Wu": torch.empty(N, K, device="cuda"), "bg": torch.empty(N, device="cuda"), "bu": torch.empty(N, device="cuda")}
    omc.omc_gated_linear_backward(layer.R, sg, su, X, Wg, Wu, *(gradients[n] for n in differences.NAMES), ws)
    for name, direction in layer.directions().items():
        layer.compare(name, gradients[name], direction, *(objective(*layer.moved(name, direction, s)) for s in (1, -1)))
