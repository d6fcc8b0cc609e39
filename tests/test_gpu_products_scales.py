"""Codes of values that lie halfway by their row's scale, where the last place of the scale decides: in every kernel that rounds."""
import pytest
import torch

import products_ref as ref
from paper_2205_03494_amd import omc
from test_products_scales_host import halves, quotients

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("by_columns", [False, True])
@pytest.mark.parametrize("length", [4, 300, 1500, 5000, 9000])      # along rows in a lane, a wave, a workgroup, twice; along columns in one launch and in three
def test_quantize(length, by_columns, dtype):
    x = torch.zeros(640, length)
    x[:, -4:] = halves()
    x = x.to(dtype).cuda()
    codes = torch.empty(640, -(-length // 128) * 128, dtype=torch.uint8, device="cuda")
    scales = torch.empty(640, device="cuda")
    omc.omc_i8_quantize(x.t().contiguous() if by_columns else x, codes, scales, by_columns=by_columns)
    want, want_scales = ref.i8(x)
    assert torch.equal(scales, want_scales) and torch.equal(codes, ref.padded_codes(want))
    assert not torch.equal(want, quotients(x)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [1, 16, 640])
def test_linear(M, dtype):
    """Weights of ones along the diagonal: Y is what the codes stand for."""
    x = halves().to(dtype).cuda()
    one = torch.ones(4, device="cuda")
    w = ref.padded_codes(torch.eye(4, device="cuda"))
    want, scales = ref.i8(x)
    Y = torch.empty(640, 4, device="cuda")
    ws = torch.empty(max(16, omc.omc_i8_linear_workspace_bytes(M, 4, 4)), dtype=torch.uint8, device="cuda")
    for first in range(0, 640, M):
        omc.omc_i8_linear(x[first:first + M], w, one, None, Y[first:first + M], ws)
    assert torch.equal(Y, want.float() * scales[:, None])
