"""A gradient's bits follow from the sizes alone: whichever others are asked for beside it, it is the same."""
import pytest
import torch

from paper_2205_03494_amd import omc

pytestmark = pytest.mark.gpu

# Few and many rows of dX, of dW; batches that are long for the matrix; results of few tiles; roundings of few and many tiles with and without X's.
SHAPES = [(1, 64, 96), (20, 64, 64), (32, 1024, 4096), (20, 4096, 1024), (8192, 64, 64), (65536, 64, 64), (50001, 33, 20), (3000, 300, 200), (4096, 1024, 4096),
          (4003, 1000, 4091), (12000, 7000, 65), (300, 520, 70), (40000, 128, 2048), (20, 8192, 8192), (8192, 20, 30)]


def mx4(values):
    rows, cols = values.shape
    codes, scales = (torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (omc.omc_mx4_code_bytes, omc.omc_mx4_scale_bytes))
    omc.omc_mx4_quantize(values, codes, scales)
    return codes, scales


def backward_of(M, N, K, dtype):
    """gradients(names) of a layer, the same inputs every time.  Blocks of 32 along the contractions are of sizes up to 2^12 apart in either operand, so that fp32 sums of their products round (4-bit values of one
    size would add up exactly, in any order)."""
    g = torch.Generator("cuda").manual_seed(M + N + K)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    sizes = lambda n: torch.exp2(torch.randint(-6, 7, (n // 32 + 1,), device="cuda", generator=g).float()).repeat_interleave(32)[:n]
    x, dy = (normal(M, K) * sizes(M)[:, None]).to(dtype), (normal(M, N) * sizes(M)[:, None] * sizes(N)).to(dtype)
    weights = mx4(normal(K, N) * sizes(N))
    ws = torch.empty(omc.omc_mx4_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")

    def gradients(*wanted):
        out = {"dx": torch.full((M, K), 7.0, device="cuda"), "dw": torch.full((K, N), 7.0, device="cuda"), "dbias": torch.full((N,), 7.0, device="cuda")}
        out = {n: t for n, t in out.items() if n in wanted}
        omc.omc_mx4_linear_backward(dy, x if "dw" in wanted else None, *(weights if "dx" in wanted else (None, None)), out.get("dx"), out.get("dw"), out.get("dbias"), ws)
        return out
    return gradients


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_a_products_gradient_is_the_same_whatever_is_asked_for_beside_it(M, N, K, dtype):
    gradients = backward_of(M, N, K, dtype)
    whole = gradients("dx", "dw", "dbias")
    for wanted in (("dx",), ("dw",), ("dx", "dw"), ("dx", "dbias"), ("dw", "dbias")):
        for name, got in gradients(*wanted).items():
            assert name == "dbias" or torch.equal(got, whole[name]), (name, "beside", wanted)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_dbias_is_the_same_whatever_is_asked_for_beside_it(M, N, K, dtype):
    gradients = backward_of(M, N, K, dtype)
    whole = gradients("dx", "dw", "dbias")["dbias"]
    for wanted in (("dbias",), ("dx", "dbias"), ("dw", "dbias")):
        assert torch.equal(gradients(*wanted)["dbias"], whole), wanted
