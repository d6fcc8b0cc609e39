"""Products on 8-bit integers and the gated layer without a GPU: sizes, and what they refuse before anything is enqueued."""
import pytest
import torch

import products_ref as ref
from paper_2205_03494_amd import omc

NULL, FORMAT, SIZE, ALIGN, WORKSPACE, OPT = 1, 2, 3, 4, 5, 6
P = 1 << 20      # any address that is aligned; nothing is read


def test_sizes():
    for rows, cols in ((1, 1), (3, 128), (5, 129), (1000, 4096), (1 << 24, 64)):
        assert omc.omc_i8_code_bytes(rows, cols) == rows * -(-cols // 128) * 128
    for rows, cols in ((0, 1), (1, 0), ((1 << 24) + 1, 1), (1, (1 << 24) + 1), (1 << 24, 1 << 14)):
        assert omc.omc_i8_code_bytes(rows, cols) == 0
        for size in (omc.omc_i8_gemm_workspace_bytes, omc.omc_i8_linear_workspace_bytes, omc.omc_i8_gated_linear_workspace_bytes,
                     omc.omc_gated_linear_workspace_bytes, omc.omc_gated_linear_backward_workspace_bytes):
            assert size(rows, cols, 64) == size(64, rows, cols) == 0
    assert omc.omc_i8_linear_workspace_bytes(64, 64, 131072) == 0 and omc.omc_i8_linear_workspace_bytes(64, 64, 131071) > 0
    assert omc.omc_gated_linear_backward_workspace_bytes((1 << 22) + 1, 64, 64) == 0


def test_the_reference_rounds_as_the_definition_says():
    x = torch.tensor([[127.0, 2.5, 3.5, -0.5, -1.5, 0.49, 126.51], [0.0] * 7, [1.0, float("inf")] + [0.0] * 5])
    codes, scales = ref.i8(x)
    assert codes[0].tolist() == [127.0, 2.0, 4.0, 0.0, -2.0, 0.0, 127.0]
    assert scales[:2].tolist() == [1.0, 0.0] and torch.isnan(scales[2]) and not codes[1:].any()


def test_the_references_gates_have_their_slopes():
    g = torch.linspace(-9, 9, 181, dtype=torch.float64)
    for kind in (ref.SIGMOID, ref.SWISH, ref.GELU):
        value, slope = ref.gate(g, kind)
        d = (ref.gate(g + 1e-4, kind)[0] - ref.gate(g - 1e-4, kind)[0]) / 2e-4
        assert (slope - d).abs().max() < 1e-8
        assert slope.abs().max() <= ref.STEEPEST[kind]
        curve = (ref.gate(g + 1e-4, kind)[1] - ref.gate(g - 1e-4, kind)[1]).abs().max() / 2e-4
        assert curve <= ref.CURVED[kind] * (1 + 1e-3)


CALLS = {
    "i8_quantize": dict(x=P, type=1, rows=8, cols=64, ldx=64, by_columns=0, codes=P, scales=P, values=P, ldv=64, stream=None),
    "i8_gemm": dict(ac=P, as_=P, bc=P, bs=P, bias=P, c=P, type=0, ldc=96, M=512, N=96, K=64, ws=P, ws_bytes=1 << 40, stream=None),
    "i8_linear": dict(x=P, xtype=1, ldx=64, wc=P, ws_=P, bias=P, y=P, ytype=0, ldy=96, M=512, N=96, K=64, ws=P, ws_bytes=1 << 40, stream=None),
    "i8_gated": dict(x=P, xtype=1, ldx=64, gc=P, gs=P, uc=P, us=P, bg=P, bu=P, gate=1, h=P, htype=0, ldh=96, M=512, N=96, K=64, ws=P,
                     ws_bytes=1 << 40, stream=None),
    "gated": dict(x=P, xtype=1, ldx=64, wg=P, wu=P, wtype=1, ldw=64, bg=P, bu=P, gate=0, h=P, htype=0, ldh=96, sg=P, su=P, lds=96, M=512, N=96,
                  K=64, ws=P, ws_bytes=1 << 40, stream=None),
    "gated_backward": dict(dh=P, htype=1, lddh=96, sg=P, su=P, lds=96, x=P, xtype=1, ldx=64, wg=P, wu=P, wtype=1, ldw=64, dx=P, dxtype=0, lddx=64,
                           dwg=P, dwu=P, dbg=P, dbu=P, M=512, N=96, K=64, ws=P, ws_bytes=1 << 40, stream=None),
}
REFUSED = [
    ("i8_quantize", NULL, [dict(x=None), dict(codes=None), dict(scales=None)]),
    ("i8_quantize", FORMAT, [dict(type=2), dict(type=-1)]),
    ("i8_quantize", SIZE, [dict(rows=0), dict(cols=0), dict(cols=(1 << 24) + 1), dict(ldx=63), dict(ldv=63)]),
    ("i8_quantize", ALIGN, [dict(x=P + 1), dict(values=P + 1), dict(codes=P + 8), dict(scales=P + 2), dict(type=0, x=P + 2)]),
    ("i8_gemm", NULL, [dict(ac=None), dict(as_=None), dict(bc=None), dict(bs=None), dict(c=None)]),
    ("i8_gemm", FORMAT, [dict(type=7)]),
    ("i8_gemm", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldc=95), dict(K=131072)]),
    ("i8_gemm", ALIGN, [dict(ac=P + 8), dict(bc=P + 4), dict(as_=P + 2), dict(bs=P + 1), dict(bias=P + 2), dict(c=P + 2)]),
    ("i8_linear", NULL, [dict(x=None), dict(wc=None), dict(ws_=None), dict(y=None)]),
    ("i8_linear", FORMAT, [dict(xtype=2), dict(ytype=3)]),
    ("i8_linear", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldx=63), dict(ldy=95), dict(K=131072, ldx=1 << 20)]),
    ("i8_linear", ALIGN, [dict(x=P + 1), dict(wc=P + 8), dict(ws_=P + 2), dict(bias=P + 1), dict(y=P + 2), dict(ws=P + 4)]),
    ("i8_linear", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_i8_linear_workspace_bytes(512, 96, 64) - 1)]),
    ("i8_gated", NULL, [dict(x=None), dict(gc=None), dict(gs=None), dict(uc=None), dict(us=None), dict(h=None)]),
    ("i8_gated", OPT, [dict(gate=3), dict(gate=-1)]),
    ("i8_gated", FORMAT, [dict(xtype=2), dict(htype=3)]),
    ("i8_gated", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldx=63), dict(ldh=95), dict(K=131072, ldx=1 << 20)]),
    ("i8_gated", ALIGN, [dict(x=P + 1), dict(gc=P + 8), dict(uc=P + 4), dict(gs=P + 2), dict(us=P + 1), dict(bg=P + 1), dict(bu=P + 2), dict(h=P + 2), dict(ws=P + 4)]),
    ("i8_gated", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_i8_gated_linear_workspace_bytes(512, 96, 64) - 1)]),
    ("gated", NULL, [dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(sg=None), dict(su=None)]),
    ("gated", FORMAT, [dict(xtype=2), dict(wtype=2), dict(htype=-1)]),
    ("gated", OPT, [dict(gate=3), dict(gate=-1)]),
    ("gated", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(ldx=63), dict(ldw=63), dict(ldh=95), dict(lds=95), dict(M=(1 << 22) + 1)]),
    ("gated", ALIGN, [dict(x=P + 1), dict(wg=P + 1), dict(wu=P + 1), dict(wtype=0, wg=P + 2), dict(bg=P + 1), dict(bu=P + 2), dict(h=P + 2), dict(sg=P + 1), dict(su=P + 1), dict(ws=P + 8)]),
    ("gated", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_gated_linear_workspace_bytes(512, 96, 64) - 1)]),
    ("gated_backward", NULL, [dict(dh=None), dict(sg=None), dict(su=None), dict(dwg=None), dict(dwu=None), dict(wg=None), dict(wu=None), dict(x=None),
                              dict(dx=None, dwg=None, dwu=None, dbg=None, dbu=None)]),
    ("gated_backward", FORMAT, [dict(htype=2), dict(xtype=2), dict(wtype=-1), dict(dxtype=2)]),
    ("gated_backward", SIZE, [dict(M=0), dict(N=0), dict(K=0), dict(lddh=95), dict(lds=95), dict(ldx=63), dict(ldw=63), dict(lddx=63), dict(N=(1 << 22) + 1, lddh=1 << 30, lds=1 << 30)]),
    ("gated_backward", ALIGN, [dict(dh=P + 1), dict(sg=P + 1), dict(su=P + 1), dict(x=P + 1), dict(wg=P + 1), dict(wu=P + 1), dict(dx=P + 2), dict(dwg=P + 2), dict(dwu=P + 1), dict(dbg=P + 2),
                               dict(dbu=P + 1), dict(ws=P + 8)]),
    ("gated_backward", WORKSPACE, [dict(ws=None), dict(ws_bytes=0), dict(ws_bytes=omc.omc_gated_linear_backward_workspace_bytes(512, 96, 64) - 1)]),
]


@pytest.mark.parametrize("fn,want,changes", REFUSED, ids=[f"{f}-{w}" for f, w, _ in REFUSED])
def test_refusals(fn, want, changes):
    for change in changes:
        args = dict(CALLS[fn])
        for k, v in change.items():
            assert k in args
            args[k] = v
        assert getattr(omc, "_" + fn)(*args.values()) == want, change


def test_binding_refuses_before_the_library():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device matrix"):
        omc.omc_i8_quantize(x, torch.zeros(512, dtype=torch.uint8), torch.zeros(4))
    with pytest.raises(ValueError, match="device matrix"):
        omc.omc_gated_linear(x, x, x, None, None, omc.OMC_GATE_SWISH, x, None, None, None)
