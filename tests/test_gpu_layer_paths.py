"""Ways through the layer's kernels that sizes or outputs asked for alone lead to: roundings of both directions without values, rows that are not finite on the way back, gradients larger than the caches."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
from paper_2205_03494_amd import omc
from test_gpu_layer import BF16, F32, SHAPES, buffers, check, empty, guarded, inputs, norm_inputs, random_codes, random_mx4, special, tensor, to_dev, untouched, values_on_device, workspace

pytestmark = pytest.mark.gpu


# More than 256 tiles of 256 x 128 too, which are then taken whole; fewer are cut into four.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad", SHAPES + [(1030, 8200, 1), (255, 33000, 0), (70000, 128, 0)])
@pytest.mark.parametrize("make", [inputs, special])
def test_both_directions_from_one_read(rows, cols, pad, dtype, make):
    x = tensor(make(rows, cols, rows * 1000 + cols + 1), dtype, pad)
    x64 = ref.as64(x)
    (cw, sw, c, s), (ctw, stw, ct, st) = buffers(rows, cols), buffers(cols, rows)
    omc.omc_mx4_quantize(x, c, s, ct, st)
    for got_c, got_s, of in ((c, s, x64), (ct, st, x64.T)):
        codes, scales, _ = ref.quantize(of)
        assert np.array_equal(got_s.cpu().numpy().reshape(len(of), -1), scales)
        assert np.array_equal(got_c.cpu().numpy().reshape(len(of), -1), codes)
    for whole, part in ((cw, c), (sw, s), (ctw, ct), (stw, st)):
        guarded(whole, part)


def finite_where(got, want, bound):
    """Finite results are checked; what is not finite in 64 bits is the same here."""
    got = ref.as64(got)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    assert (np.abs(got - want)[~odd] <= (bound + ref.rounding(np.abs(want) + bound, F32))[~odd]).all()


# few rows of dX, of dW; both products together in either tile; apart
@pytest.mark.parametrize("M,N,K", [(20, 96, 300), (300, 520, 70), (700, 100, 20), (2100, 128, 384), (2990, 1100, 1555), (20, 8192, 100), (8192, 300, 20)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_linear_backward_of_values_that_are_not_finite(M, N, K, dtype):
    x, dy = inputs(M, K, 1), inputs(M, N, 2, 1e-3)
    x[M // 2, K // 3] = np.inf
    x[M - 1, K - 1] = np.nan
    dy[M // 3, N // 2] = np.nan
    dy[M // 5, 3] = -np.inf
    xd, dyd = tensor(x, dtype), tensor(dy, dtype)
    wc, wsc, w = random_mx4(K, N, 3)
    x64, dy64 = ref.as64(xd), ref.as64(dyd)
    dyq, dyt, xt = ref.quantize(dy64)[2], ref.quantize(dy64.T)[2], ref.quantize(x64.T)[2]
    dx, dw, dbias = torch.empty(M, K, device="cuda"), torch.empty(K, N, device="cuda"), torch.empty(N, device="cuda")
    omc.omc_mx4_linear_backward(dyd, xd, to_dev(wc), to_dev(wsc), dx, dw, dbias, workspace(omc.omc_mx4_linear_backward_workspace_bytes(M, N, K))[1])
    with np.errstate(invalid="ignore"):
        check(dx, dyq @ w.T, ref.product_bound(dyq, w, N), F32)
        check(dw, xt @ dyt.T, ref.product_bound(xt, dyt, M), F32)
        finite_where(dbias, dy64.sum(0), (64 + M / 128) * 2.0 ** -24 * np.abs(dy64).sum(0))
    assert np.isnan(ref.as64(dx)).any(1).sum() == 2 and np.isinf(ref.as64(dbias)).sum() == 1


@pytest.mark.parametrize("rows,cols", [(12, 300), (40, 64), (9, 1000), (130, 2056), (6, 5001), (3, 16385)])
@pytest.mark.parametrize("x_type,dy_type", [(F32, F32), (BF16, BF16)])
def test_rows_of_a_norms_gradient_that_are_not_finite_stay_alone(rows, cols, x_type, dy_type):
    x, gamma, _ = norm_inputs(rows, cols, 3)
    dy = inputs(rows, cols, 4, 1e-2)
    x[rows - 1, 7] = np.inf                      # the whole row of x, mean and rstd
    dy[1, cols - 1] = np.nan                     # of one column alone
    xd, dyd = tensor(x, x_type), tensor(dy, dy_type)
    x64, dy64 = ref.as64(xd), ref.as64(dyd)
    y, mean, rstd = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    g = torch.from_numpy(gamma).cuda()
    omc.omc_layer_norm(xd, g, None, 1e-5, y, mean, rstd)
    dx, dg, db = torch.empty(rows, cols, device="cuda", dtype=x_type), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    omc.omc_layer_norm_backward(dyd, xd, g, mean, rstd, dx, dg, db, workspace(omc.omc_layer_norm_backward_workspace_bytes(rows, cols))[1])
    bad = np.isnan(ref.as64(dx))
    assert bad.all(1).tolist() == [i in (1, rows - 1) for i in range(rows)] and bad.any(1).tolist() == bad.all(1).tolist()
    assert np.isnan(ref.as64(dg)).all()          # a sum over all rows
    assert np.isnan(ref.as64(db)).tolist() == [c == cols - 1 for c in range(cols)]
    finite_where(db, dy64.sum(0), (64 + rows / 32) * 2.0 ** -24 * np.abs(dy64).sum(0))
    clean = [i for i in range(rows) if i not in (1, rows - 1)]
    m64, r64 = ref.as64(mean)[clean], ref.as64(rstd)[clean]
    want = ref.layer_norm_backward(dy64[clean], x64[clean], gamma.astype(np.float64), m64, r64)[0]
    alone = torch.empty(len(clean), cols, device="cuda", dtype=x_type)
    omc.omc_layer_norm_backward(dyd[clean], xd[clean], g, mean[clean], rstd[clean], alone, None, None, workspace(omc.omc_layer_norm_backward_workspace_bytes(len(clean), cols))[1])
    assert torch.equal(alone, dx[clean])         # rows are sums of their own
    assert np.allclose(ref.as64(alone), want, rtol=2.0 ** -7, atol=2.0 ** -7 * np.abs(want).max())


# dX of 32 MB and more in bf16, whose rows are whole cache lines, beside dW in the same launch, in either tile; whole tiles and not.
LARGE_GRADIENTS = [(8192, 1024, 4096), (6000, 300, 4096), (8192, 128, 2048), (4100, 64, 4096)]


@pytest.mark.parametrize("dx_type", [F32, BF16])
@pytest.mark.parametrize("M,N,K", LARGE_GRADIENTS)
def test_a_gradient_larger_than_the_caches_beside_the_weights(M, N, K, dx_type):
    g = torch.Generator("cuda").manual_seed(M + N + K)
    x, dy = torch.randn(M, K, device="cuda", generator=g).to(BF16), torch.randn(M, N, device="cuda", generator=g).to(BF16)
    w = [torch.from_numpy(a.reshape(-1)).cuda() for a in random_codes(K, N, 1)]
    mx4 = lambda rows, cols: [torch.empty(f(rows, cols), dtype=torch.uint8, device="cuda") for f in (omc.omc_mx4_code_bytes, omc.omc_mx4_scale_bytes)]
    dyq, dyt, xt = mx4(M, N), mx4(N, M), mx4(K, M)
    omc.omc_mx4_quantize(dy, *dyq, *dyt)
    omc.omc_mx4_quantize(x, None, None, *xt)
    dxw, dx = empty(M, K, dx_type)
    dw, dbias = torch.full((K, N), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
    whole, ws = workspace(omc.omc_mx4_linear_backward_workspace_bytes(M, N, K))
    omc.omc_mx4_linear_backward(dy, x, *w, dx, dw, dbias, ws)
    for got, a, b, rows, cols, along, dtype in ((dx, dyq, w, M, K, N, dx_type), (dw, xt, dyt, K, N, M, F32)):
        av, bv = values_on_device(*a, rows, along), values_on_device(*b, cols, along)
        want, bound = av @ bv.t(), ref.product_bound_of(av.abs() @ bv.abs().t(), along)
        assert ((got.double() - want).abs() <= bound + (want.abs() + bound) * (2.0 ** -8 if dtype is BF16 else 2.0 ** -23)).all()
    assert ((dbias.double() - dy.double().sum(0)).abs() <= (64 + M / 128) * 2.0 ** -24 * dy.double().abs().sum(0)).all()
    untouched(dxw, K)
    guarded(whole, ws)
