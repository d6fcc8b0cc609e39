"""Every tile and every cut of the products, results larger than the caches, unaligned slices, far rows, values that are not finite on the way."""
import math

import pytest
import torch

import products_ref as ref
from paper_2205_03494_amd import omc
from test_gpu_products import BF16, F32, GATES, i8_weights, layer, out, rand, space, untouched

pytestmark = pytest.mark.gpu

_tile = omc._lib.omc_internal_product_tile
_pair = omc._lib.omc_internal_product_pair_tile
I8, I8_GATED, GATED, DX, DW = range(5)


def stages(n, of=64):
    return -(-n // of)


def tile_of(kind, M, N, K):
    if kind in (I8, I8_GATED):
        c = _tile(kind, M, N, stages(K, 128))
    elif kind == GATED:
        c = _tile(kind, M, N, stages(K))
    elif kind == DX:
        c = _tile(kind, M, K, 2 * stages(N))
    else:
        c = _tile(kind, 128 * stages(N), K, stages(M))
    return c % 16, c // 16


I8_CASES = [(0, 1, 1818, 7944, 21), (1, 1, 3668, 1538, 20), (1, 4, 8629, 66, 8985), (2, 1, 8996, 265, 22), (2, 8, 2204, 71, 6736), (3, 1, 35, 34, 21), (3, 8, 35, 34, 1996), (0, 1, 4096, 4096, 512),
            (3, 16, 33, 33, 64000)]
I8_GATED_CASES = [(0, 1, 4072, 1936, 20), (1, 1, 900, 6386, 141), (1, 4, 8553, 34, 5566), (2, 1, 268, 4834, 20), (2, 8, 65, 1093, 8709), (3, 1, 35, 34, 21), (3, 4, 36, 34, 1751)]
GATED_CASES = [(0, 1, 6411, 1043, 20), (0, 4, 268, 3404, 6889), (1, 1, 443, 8122, 21), (1, 4, 8328, 34, 4964), (2, 1, 66, 8840, 21), (2, 8, 2054, 33, 4930), (3, 1, 35, 34, 21), (3, 4, 33, 34, 772)]
DX_CASES = [(0, 1, 1815, 34, 7988), (0, 8, 130, 6597, 5609), (1, 1, 4376, 33, 2697), (1, 4, 8294, 7085, 21), (2, 1, 8980, 38, 193), (2, 16, 66, 4420, 1105), (3, 1, 1841, 34, 20), (3, 8, 34, 942, 20)]
DW_CASES = [(0, 1, 67, 8295, 4548), (1, 1, 3857, 8319, 200), (1, 2, 8119, 8508, 70), (2, 1, 132, 8430, 359), (2, 16, 7727, 1027, 66), (3, 1, 34, 942, 20), (3, 8, 1841, 34, 20)]
PAIRS = [(0, 903, 348, 7508), (1, 3006, 1755, 586), (2, 66, 34, 7328), (3, 35, 34, 21)]


@pytest.mark.parametrize("c_type", [F32, BF16])
@pytest.mark.parametrize("tile,splits,M,N,K", I8_CASES)
def test_i8_gemm_in_every_tile(tile, splits, M, N, K, c_type):
    codes, scales = ref.i8(rand(M, K, 4))
    w_codes, w_scales, w = i8_weights(N, K, 5)
    bias = torch.randn(N, device="cuda", generator=torch.Generator("cuda").manual_seed(6))
    wide, C = out(M, N, c_type)
    whole, ws = space(omc.omc_i8_gemm_workspace_bytes(M, N, K))
    omc.omc_i8_gemm(ref.padded_codes(codes), scales, w, w_scales, bias, C, K, ws)
    ref.check(C, *ref.i8_product(codes, scales, w_codes, w_scales, bias))
    untouched(wide, M, N)
    assert (whole[-64:] == 0xFF).all()


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("tile,splits,M,N,K", I8_GATED_CASES)
def test_i8_gated_in_every_tile(tile, splits, M, N, K, gate):
    X = rand(M, K, 12)
    (gc, gs, wg), (uc, us, wu) = i8_weights(N, K, 13), i8_weights(N, K, 14)
    bg = torch.randn(N, device="cuda", generator=torch.Generator("cuda").manual_seed(15))
    codes, scales = ref.i8(X)
    want = ref.gated(*ref.i8_product(codes, scales, gc, gs, bg), *ref.i8_product(codes, scales, uc, us), gate)["h"]
    for h_type in (F32, BF16):
        wide, H = out(M, N, h_type)
        whole, ws = space(omc.omc_i8_gated_linear_workspace_bytes(M, N, K))
        omc.omc_i8_gated_linear(X, wg, gs, wu, us, bg, None, gate, H, ws)
        ref.check(H, *want)
        untouched(wide, M, N)
        assert (whole[-64:] == 0xFF).all()


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("tile,splits,M,N,K", GATED_CASES)
def test_gated_in_every_tile(tile, splits, M, N, K, gate):
    X, Wg, Wu, bg, bu = layer(M, N, K, BF16, BF16, 0)
    want = ref.gated(*ref.product(X.double(), Wg.double(), bg), *ref.product(X.double(), Wu.double(), None), gate)
    for h_type in (F32, BF16):
        (wide, H), (wide_g, sg), (wide_u, su) = out(M, N, h_type), out(M, N, BF16), out(M, N, BF16)
        whole, ws = space(omc.omc_gated_linear_workspace_bytes(M, N, K))
        omc.omc_gated_linear(X, Wg, Wu, bg, None, gate, H, sg, su, ws)
        for name, got in (("h", H), ("slope_g", sg), ("slope_u", su)):
            ref.check(got, *want[name], name)
        for w in (wide, wide_g, wide_u):
            untouched(w, M, N)
        assert (whole[-64:] == 0xFF).all()


@pytest.mark.parametrize("M,N,K", [c[2:] for c in DX_CASES + DW_CASES] + [p[1:] for p in PAIRS])
def test_backward_in_every_tile(M, N, K):
    X, Wg, Wu, _, _ = layer(M, N, K, BF16, BF16, 0)
    dH, sg, su = rand(M, N, 25, BF16, 0, 0.01), rand(M, N, 26, BF16), rand(M, N, 27, BF16)
    dg, du = dH.float() * sg.float(), dH.float() * su.float()
    rg, ru = ref.rounded(dg), ref.rounded(du)
    want_x = ref.product(torch.cat((rg, ru), 1), torch.cat((Wg.double(), Wu.double()), 0).t())
    for dx_type in (F32, BF16):
        wide, dX = out(M, K, dx_type)
        dWg, dWu, dbg, dbu = torch.full((N, K), 7.0, device="cuda"), torch.full((N, K), 7.0, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        whole, ws = space(omc.omc_gated_linear_backward_workspace_bytes(M, N, K))
        omc.omc_gated_linear_backward(dH, sg, su, X, Wg, Wu, dX, dWg, dWu, dbg, dbu, ws)
        ref.check(dX, *want_x, "dX")
        untouched(wide, M, K)
        assert (whole[-64:] == 0xFF).all()
        alone = torch.empty(M, K, dtype=dx_type, device="cuda")
        omc.omc_gated_linear_backward(dH, sg, su, None, Wg, Wu, alone, None, None, None, None, ws)
        assert torch.equal(alone, dX)
    for got, d in ((dWg, rg), (dWu, ru)):
        ref.check(got, *ref.product(d.t(), X.double().t()), "dW")
    for got, d in ((dbg, dg.double()), (dbu, du.double())):
        ref.check(got, d.sum(0), (M + 1) * ref.U * d.abs().sum(0), "db")
    a, b = torch.empty_like(dWg), torch.empty_like(dWu)
    omc.omc_gated_linear_backward(dH, sg, su, X, None, None, None, a, b, None, None, ws)
    assert torch.equal(a, dWg) and torch.equal(b, dWu)


@pytest.mark.parametrize("keep", [False, True])
def test_results_larger_than_the_caches(keep):
    M, N, K = 4352, 4096, 64            # 17 whole tiles of 256 rows: all results go past the caches
    X, Wg, Wu, bg, bu = layer(M, N, K, BF16, BF16, 0)
    H = torch.empty(M, N, dtype=BF16, device="cuda")
    sg, su = (torch.empty_like(H), torch.empty_like(H)) if keep else (None, None)
    ws = torch.empty(omc.omc_gated_linear_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    omc.omc_gated_linear(X, Wg, Wu, bg, bu, omc.OMC_GATE_SWISH, H, sg, su, ws)
    want = ref.gated(*ref.product(X.double(), Wg.double(), bg), *ref.product(X.double(), Wu.double(), bu), omc.OMC_GATE_SWISH)
    ref.check(H, *want["h"])
    if keep:
        ref.check(sg, *want["slope_g"])
        ref.check(su, *want["slope_u"])
    codes, scales = ref.i8(X)
    (gc, gs, wg), (uc, us, wu) = i8_weights(N, K, 13), i8_weights(N, K, 14)
    ws = torch.empty(omc.omc_i8_gated_linear_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    omc.omc_i8_gated_linear(X, wg, gs, wu, us, bg, bu, omc.OMC_GATE_GELU, H, ws)
    ref.check(H, *ref.gated(*ref.i8_product(codes, scales, gc, gs, bg), *ref.i8_product(codes, scales, uc, us, bu), omc.OMC_GATE_GELU)["h"])


def test_plain_results_larger_than_the_caches():
    M = N = 8192
    codes, scales = ref.i8(rand(M, 40, 4))
    w_codes, w_scales, w = i8_weights(N, 40, 5)
    C = torch.empty(M, N, dtype=BF16, device="cuda")
    omc.omc_i8_gemm(ref.padded_codes(codes), scales, w, w_scales, None, C, 40, space(omc.omc_i8_gemm_workspace_bytes(M, N, 40))[1])
    ref.check(C, *ref.i8_product(codes, scales, w_codes, w_scales))


@pytest.mark.parametrize("M", [5, 70, 300])
def test_slices_that_begin_anywhere(M):
    """Bases off every alignment but their elements', row strides odd."""
    N, K = 130, 192

    def part(rows, cols, seed, dtype):
        return rand(rows, cols + 1, seed, dtype, 2)[:, 1:]

    def hole(rows, cols, dtype):
        wide, t = out(rows, cols + 1, dtype, 2)
        return wide, t[:, 1:]
    for dtype in (BF16, F32):
        X, Wg, Wu = part(M, K, 40, dtype), part(N, K, 41, dtype), part(N, K, 42, dtype)
        (wide, H), (_, sg), (_, su) = hole(M, N, dtype), hole(M, N, BF16), hole(M, N, BF16)
        omc.omc_gated_linear(X, Wg, Wu, None, None, omc.OMC_GATE_GELU, H, sg, su, space(omc.omc_gated_linear_workspace_bytes(M, N, K))[1])
        want = ref.gated(*ref.product(ref.rounded(X), ref.rounded(Wg)), *ref.product(ref.rounded(X), ref.rounded(Wu)), omc.OMC_GATE_GELU)
        for name, got in (("h", H), ("slope_g", sg), ("slope_u", su)):
            ref.check(got, *want[name], name)
        assert (wide[:, 0] == 7.0).all() and (wide[:, N + 1:] == 7.0).all()
        dH, (wide, dX) = part(M, N, 43, dtype), hole(M, K, dtype)
        dWg, dWu = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
        omc.omc_gated_linear_backward(dH, sg, su, X, Wg, Wu, dX, dWg, dWu, None, None, space(omc.omc_gated_linear_backward_workspace_bytes(M, N, K))[1])
        rg, ru = ref.rounded(dH.float() * sg.float()), ref.rounded(dH.float() * su.float())
        ref.check(dX, *ref.product(torch.cat((rg, ru), 1), torch.cat((ref.rounded(Wg), ref.rounded(Wu)), 0).t()), "dX")
        ref.check(dWg, *ref.product(rg.t(), ref.rounded(X).t()), "dWg")
        ref.check(dWu, *ref.product(ru.t(), ref.rounded(X).t()), "dWu")
        assert (wide[:, 0] == 7.0).all() and (wide[:, K + 1:] == 7.0).all()
        w_codes, w_scales, w = i8_weights(N, K, 44)
        wide, Y = hole(M, N, dtype)
        omc.omc_i8_linear(X, w, w_scales, None, Y, space(omc.omc_i8_linear_workspace_bytes(M, N, K))[1])
        ref.check(Y, *ref.i8_product(*ref.i8(X), w_codes, w_scales))
        assert (wide[:, 0] == 7.0).all() and (wide[:, N + 1:] == 7.0).all()


@pytest.mark.parametrize("M", [6, 40])
def test_rows_far_apart(M):
    """Offsets past 32 bits: rows of inputs and results 2^27 elements apart (as they are read: 2^28 bytes), of which only the beginnings are looked at."""
    N, K, far = 48, 64, 1 << 27
    room = torch.empty(M * far, dtype=BF16, device="cuda").view(M, far)
    X, H, sg, su, dX = (room[:, i * 64:i * 64 + n] for i, n in enumerate((K, N, N, N, K)))
    x, Wg, Wu, bg, bu = layer(M, N, K, BF16, BF16, 0)
    X.copy_(x)
    omc.omc_gated_linear(X, Wg, Wu, bg, bu, omc.OMC_GATE_SWISH, H, sg, su, space(omc.omc_gated_linear_workspace_bytes(M, N, K))[1])
    want = ref.gated(*ref.product(x.double(), Wg.double(), bg), *ref.product(x.double(), Wu.double(), bu), omc.OMC_GATE_SWISH)
    for name, got in (("h", H), ("slope_g", sg), ("slope_u", su)):
        ref.check(got.clone(), *want[name], name)
    dWg, dWu = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
    omc.omc_gated_linear_backward(H, sg, su, X, Wg, Wu, dX, dWg, dWu, None, None, space(omc.omc_gated_linear_backward_workspace_bytes(M, N, K))[1])
    rg, ru = ref.rounded(H.float() * sg.float()), ref.rounded(H.float() * su.float())
    ref.check(dX.clone(), *ref.product(torch.cat((rg, ru), 1), torch.cat((Wg.double(), Wu.double()), 0).t()), "dX")
    ref.check(dWg, *ref.product(rg.t(), x.double().t()), "dWg")
    w_codes, w_scales, w = i8_weights(N, K, 44)
    omc.omc_i8_linear(X, w, w_scales, None, H, space(omc.omc_i8_linear_workspace_bytes(M, N, K))[1])
    ref.check(H.clone(), *ref.i8_product(*ref.i8(x), w_codes, w_scales))


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("M", [4, 80])
def test_gates_far_out_and_values_that_are_not_finite(M, gate):
    """g = x bg-wise: Wg is zero, so that g is the bias, from one end of fp32 to the other; u is one."""
    ends = [0.0, -0.0, 1e-30, 1.0, -1.0, 5.0, -5.0, 9.0, -9.0, 20.0, -20.0, 87.0, -87.0, 89.0, -89.0, 104.0, -104.0, 1e4, -1e4, 1e19, -1e19, 3e38, -3e38, math.inf, -math.inf, math.nan]
    g = torch.tensor(ends, device="cuda")
    N, K = len(ends), 64
    X, W = torch.ones(M, K, dtype=BF16, device="cuda"), torch.zeros(N, K, dtype=BF16, device="cuda")
    H, sg, su = torch.empty(M, N, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")
    ws = torch.empty(max(16, omc.omc_gated_linear_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    omc.omc_gated_linear(X, W, W, g, torch.ones(N, device="cuda"), gate, H, sg, su, ws)
    wide = g.double().expand(M, N)
    nothing = torch.zeros_like(wide)
    finite = torch.where(torch.isfinite(wide), wide, 0.0)
    want = ref.gated(wide, nothing, torch.ones_like(wide), nothing, gate)
    for name, got in (("h", H), ("slope_g", sg), ("slope_u", su)):
        value = want[name][0]
        # (the bound of a gate counts 1 + |g| of its roundings; beyond 2^20 it is the value's own)
        ref.check(got, value, ref.GATE * (1 + finite.abs().clamp(max=2.0 ** 20)) + 2 * ref.U * torch.where(torch.isfinite(value), value, 0.0).abs(), name)


def test_a_row_that_is_not_finite_stays_alone():
    for M, N, K in ((5, 40, 200), (90, 70, 128), (90, 70, 130)):
        X, Wg, Wu, _, _ = layer(M, N, K, BF16, BF16, 0)
        ws = torch.empty(max(omc.omc_gated_linear_workspace_bytes(M, N, K), omc.omc_gated_linear_backward_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
        both = []
        for bad in (False, True):
            if bad:
                X[2, K - 1] = math.inf
                X[3, 0] = math.nan
            H, sg, su = (torch.empty(M, N, dtype=BF16, device="cuda") for _ in range(3))
            omc.omc_gated_linear(X, Wg, Wu, None, None, omc.OMC_GATE_SIGMOID, H, sg, su, ws)
            dX = torch.empty(M, K, device="cuda")
            omc.omc_gated_linear_backward(H, sg, su, None, Wg, Wu, dX, None, None, None, None, ws)
            both.append((H, sg, su, dX))
        rest = [i for i in range(M) if i not in (2, 3)]
        for a, b in zip(*both):
            assert torch.equal(a[rest], b[rest]) and torch.isfinite(b[rest]).all()
        assert torch.isnan(both[1][0][3]).all()


def test_repeated_calls_give_the_same_bits():
    M, N, K = 700, 520, 1100
    X, Wg, Wu, bg, bu = layer(M, N, K, BF16, BF16, 0)
    ws = torch.empty(max(omc.omc_gated_linear_workspace_bytes(M, N, K), omc.omc_gated_linear_backward_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    first = None
    for fill in (0, 255, 3):
        ws.fill_(fill)
        H, sg, su = torch.empty(M, N, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")
        omc.omc_gated_linear(X, Wg, Wu, bg, bu, omc.OMC_GATE_SWISH, H, sg, su, ws)
        dX, dWg, dWu, dbg, dbu = torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        ws.fill_(fill)
        omc.omc_gated_linear_backward(H, sg, su, X, Wg, Wu, dX, dWg, dWu, dbg, dbu, ws)
        now = (H, sg, su, dX, dWg, dWu, dbg, dbu)
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now
