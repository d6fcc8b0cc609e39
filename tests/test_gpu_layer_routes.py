"""Products at the bounds between the kernel of few rows and the tiles, against 64 bits."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
from paper_2205_03494_amd import omc
from test_gpu_layer import BF16, F32, check, empty, guarded, inputs, product_is_right, random_mx4, tensor, to_dev, untouched, workspace

pytestmark = pytest.mark.gpu

FEW_AND_LONG = [(1, 33, 41000), (16, 40, 40960), (16, 40, 40961), (7, 2048, 41100), (7, 2049, 41100), (17, 33, 20480), (17, 33, 20481), (32, 300, 20577), (32, 17, 131073), (5, 1, 300000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", FEW_AND_LONG)
def test_few_rows_of_a_long_contraction(shape, dtype):
    product_is_right(*shape, dtype, 3)


@pytest.mark.parametrize("M,N,K,pad", [(16, 24, 41000, 1), (32, 65, 20500, 0), (1, 17, 60000, 3)])
def test_linear_of_few_rows_and_a_long_contraction(M, N, K, pad):
    x = tensor(inputs(M, K, 1), BF16, pad)
    wc, wsc, w = random_mx4(N, K, 2)
    bias = np.random.default_rng(3).standard_normal(N).astype(np.float32)
    whole, ws = workspace(omc.omc_mx4_linear_workspace_bytes(M, N, K))
    a = ref.quantize(ref.as64(x))[2]
    yw, y = empty(M, N, F32, pad)
    omc.omc_mx4_linear(x, to_dev(wc), to_dev(wsc), torch.from_numpy(bias).cuda(), y, ws)
    check(y, a @ w.T + bias, ref.product_bound(a, w, K) + 2.0 ** -23 * np.abs(bias), F32)
    untouched(yw, N)
    guarded(whole, ws)


@pytest.mark.parametrize("M,N,K", [(20481, 40, 32), (41000, 33, 16), (50000, 130, 20), (16, 41000, 30), (32, 20500, 100)])
def test_backward_of_a_narrow_layer_and_a_long_batch(M, N, K):
    x, dy = tensor(inputs(M, K, 5), BF16), tensor(inputs(M, N, 6, 1e-3), BF16)
    wc, wsc, w = random_mx4(K, N, 7)
    x64, dy64 = ref.as64(x), ref.as64(dy)
    dyq, dyt, xt = ref.quantize(dy64)[2], ref.quantize(dy64.T)[2], ref.quantize(x64.T)[2]
    whole, ws = workspace(omc.omc_mx4_linear_backward_workspace_bytes(M, N, K))
    dx, dw, dbias = torch.empty(M, K, device="cuda"), torch.empty(K, N, device="cuda"), torch.empty(N, device="cuda")
    omc.omc_mx4_linear_backward(dy, x, to_dev(wc), to_dev(wsc), dx, dw, dbias, ws)
    check(dx, dyq @ w.T, ref.product_bound(dyq, w, N), F32)
    check(dw, xt @ dyt.T, ref.product_bound(xt, dyt, M), F32)
    check(dbias, dy64.sum(0), (64 + M / 128) * 2.0 ** -24 * np.abs(dy64).sum(0), F32)
    guarded(whole, ws)
