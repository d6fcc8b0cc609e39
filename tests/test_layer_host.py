"""The layer's operators without a GPU: sizes, and what they refuse before anything is enqueued."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
from paper_2205_03494_amd import omc

NULL, FORMAT, SIZE, ALIGN, WORKSPACE, OPT = 1, 2, 3, 4, 5, 6
P = 1 << 20      # any address that is aligned; nothing is read


def test_sizes():
    for rows, cols in ((1, 1), (3, 32), (5, 128), (7, 129), (1000, 4096), (1 << 24, 64)):
        assert omc.omc_mx4_code_bytes(rows, cols) == rows * ref.padded(cols) // 2
        assert omc.omc_mx4_scale_bytes(rows, cols) == rows * ref.padded(cols) // 32
    for rows, cols in ((0, 1), (1, 0), ((1 << 24) + 1, 1), (1, (1 << 24) + 1), (1 << 24, 1 << 14)):
        assert omc.omc_mx4_code_bytes(rows, cols) == omc.omc_mx4_scale_bytes(rows, cols) == 0
        assert omc.omc_layer_norm_backward_workspace_bytes(rows, cols) == 0
        assert omc.omc_mx4_linear_workspace_bytes(rows, cols, 64) == omc.omc_mx4_linear_workspace_bytes(64, rows, cols) == 0
        assert omc.omc_mx4_linear_backward_workspace_bytes(rows, cols, 64) == 0
        assert omc.omc_mx4_gemm_workspace_bytes(rows, cols, 64) == 0


def test_the_reference_rounds_as_the_definition_says():
    # one block: largest 7 -> unit 1; ties to the even code, saturation
    x = np.array([[7.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -0.75, -6.9, 0.26] + [0.0] * 20])
    codes, scales, v = ref.quantize(x)
    assert v[0, :12].tolist() == [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, 0.0, 0.0, -1.0, -6.0, 0.5]
    assert scales[0].tolist() == [127, 0, 0, 0] and codes.shape == (1, 64)
    assert np.array_equal(ref.values(codes, scales, 32), v)


def status(fn, **changes):
    """Status of a call that would be fine but for the changed arguments (none of which may be fine)."""
    args = dict(CALLS[fn])
    for k, v in changes.items():
        assert k in args
        args[k] = v
    return getattr(omc, "_" + fn)(*args.values())


CALLS = {
    "mx4_quantize": dict(x=P, type=1, rows=8, cols=64, ldx=64, codes=P, scales=P, codes_t=P, scales_t=P, values=P, ldv=64, stream=None),
    "mx4_gemm": dict(ac=P, as_=P, bc=P, bs=P, bias=P, c=P, type=0, ldc=96, M=512, N=96, K=4096, ws=P, ws_bytes=1 << 40, stream=None),
    "mx4_linear": dict(x=P, xtype=1, ldx=64, wc=P, ws_=P, bias=P, y=P, ytype=0, ldy=96, M=512, N=96, K=64, ws=P, ws_bytes=1 << 40, stream=None),
    "mx4_backward": dict(dy=P, lddy=96, x=P, ldx=64, type=1, wc=P, ws_=P, dx=P, dxtype=0, lddx=64, dw=P, dbias=P, M=512, N=96, K=64, ws=P,
                         ws_bytes=1 << 40, stream=None),
    "norm": dict(x=P, xtype=0, ldx=64, gamma=P, beta=P, eps=1e-5, y=P, ytype=1, ldy=64, mean=P, rstd=P, rows=8, cols=64, stream=None),
    "norm_backward": dict(dy=P, dytype=1, lddy=64, x=P, xtype=0, ldx=64, gamma=P, mean=P, rstd=P, dx=P, lddx=64, dgamma=P, dbeta=P, rows=8,
                          cols=64, ws=P, ws_bytes=1 << 40, stream=None),
}
REFUSED = [
    ("mx4_quantize", NULL, [dict(x=None), dict(codes=None), dict(scales=None), dict(codes_t=None), dict(scales_t=None),
                            dict(codes=None, scales=None, codes_t=None, scales_t=None, values=None)]),
    ("mx4_quantize", FORMAT, [dict(type=2), dict(type=-1)]),
    ("mx4_quantize", SIZE, [dict(rows=0), dict(cols=0), dict(cols=(1 << 24) + 1), dict(rows=1 << 24, cols=1 << 14, ldx=1 << 14, ldv=1 << 14), dict(ldx=63), dict(ldv=63), dict(ldx=0)]),
    ("mx4_quantize", ALIGN, [dict(x=P + 1), dict(values=P + 1), dict(codes=P + 8), dict(scales=P + 2), dict(codes_t=P + 4), dict(scales_t=P + 1), dict(type=0, x=P + 2)]),
    ("mx4_gemm", NULL, [dict(ac=None), dict(as_=None), dict(bc=None), dict(bs=None), dict(c=None)]),
    ("mx4_gemm", FORMAT, [dict(type=7)]),
    ("mx4_gemm", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldc=95), dict(K=(1 << 24) + 1)]),
    ("mx4_gemm", ALIGN, [dict(ac=P + 8), dict(bc=P + 4), dict(as_=P + 2), dict(bs=P + 1), dict(bias=P + 2), dict(c=P + 2), dict(ws=P + 8)]),
    ("mx4_gemm", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_mx4_gemm_workspace_bytes(512, 96, 4096) - 1)]),
    ("mx4_linear", NULL, [dict(x=None), dict(wc=None), dict(ws_=None), dict(y=None)]),
    ("mx4_linear", FORMAT, [dict(xtype=2), dict(ytype=3)]),
    ("mx4_linear", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldx=63), dict(ldy=95), dict(N=(1 << 24) + 1, ldy=1 << 30)]),
    ("mx4_linear", ALIGN, [dict(x=P + 1), dict(wc=P + 8), dict(ws_=P + 2), dict(bias=P + 1), dict(y=P + 2), dict(ws=P + 4)]),
    ("mx4_linear", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_mx4_linear_workspace_bytes(512, 96, 64) - 1)]),
    ("mx4_backward", NULL, [dict(dy=None), dict(x=None), dict(wc=None), dict(ws_=None), dict(dx=None, dw=None, dbias=None)]),
    ("mx4_backward", FORMAT, [dict(type=2), dict(dxtype=2)]),
    ("mx4_backward", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(lddy=95), dict(ldx=63), dict(lddx=63)]),
    ("mx4_backward", ALIGN, [dict(dy=P + 1), dict(x=P + 1), dict(dx=P + 2), dict(dw=P + 2), dict(dbias=P + 1), dict(wc=P + 8), dict(ws=P + 8)]),
    ("mx4_backward", WORKSPACE, [dict(ws=None), dict(ws_bytes=omc.omc_mx4_linear_backward_workspace_bytes(512, 96, 64) - 1)]),
    ("norm", NULL, [dict(x=None), dict(y=None)]),
    ("norm", FORMAT, [dict(xtype=2), dict(ytype=9)]),
    ("norm", SIZE, [dict(rows=0), dict(cols=0), dict(ldx=63), dict(ldy=63)]),
    ("norm", OPT, [dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf"))]),
    ("norm", ALIGN, [dict(x=P + 2), dict(y=P + 1), dict(gamma=P + 2), dict(beta=P + 1), dict(mean=P + 2), dict(rstd=P + 3)]),
    ("norm_backward", NULL, [dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dgamma=None, dbeta=None)]),
    ("norm_backward", FORMAT, [dict(dytype=2), dict(xtype=2)]),
    ("norm_backward", SIZE, [dict(rows=0), dict(cols=0), dict(lddy=63), dict(ldx=63), dict(lddx=63)]),
    ("norm_backward", ALIGN, [dict(dy=P + 1), dict(x=P + 2), dict(dx=P + 2), dict(gamma=P + 1), dict(mean=P + 2), dict(dgamma=P + 2), dict(dbeta=P + 2), dict(ws=P + 4)]),
    ("norm_backward", WORKSPACE, [dict(ws=None), dict(ws_bytes=omc.omc_layer_norm_backward_workspace_bytes(8, 64) - 1)]),
]


@pytest.mark.parametrize("fn,want,changes", [(f, w, c) for f, w, cs in REFUSED for c in cs])
def test_refused_before_anything_is_enqueued(fn, want, changes):
    assert status(fn, **changes) == want


def test_the_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        omc.omc_mx4_quantize(x, values=x)                  # not on the device
    with pytest.raises(ValueError):
        omc.omc_layer_norm(x, None, None, 1e-5, x)


def test_every_tile_of_the_product_is_taken():
    seen = {ref.product_tile(*shape) for shape in ref.PRODUCTS}
    assert {(tile, turns) for tile, cut, turns in seen if not cut} == {(tile, turns) for tile in range(3) for turns in (False, True)}
    assert {tile for tile, cut, _ in seen if cut} == {1, 2}


def test_backward_passes_go_together_and_apart():
    assert {ref.pair_tile(M, N, K) for M, N, K, _ in ref.BACKWARD} == {-1, 1, 2} and ref.pair_tile(50001, 33, 20) == ref.pair_tile(20, 8192, 8192) == -1


def test_large_results_in_every_tile():
    assert {ref.product_tile(*shape)[0] for shape in ref.LARGE_RESULTS} == {0, 1, 2} and all(2 * M * N >= 1 << 25 and N % 64 == 0 for M, N, _ in ref.LARGE_RESULTS)
