"""Plain 64-bit forms of the products on 8-bit integers and of the gated linear layer, and how far 32-bit arithmetic may be from them."""
import math

import torch

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24                       # a rounding to fp32, relative
SIGMOID, SWISH, GELU = 0, 1, 2
STEEPEST = {SIGMOID: 0.25, SWISH: 1.1, GELU: 1.13}      # of act
CURVED = {SIGMOID: 0.0963, SWISH: 0.5, GELU: 0.798}     # most of |act''|
# A gate's value and slope in fp32 from an exact argument: exp and erfc within 8 roundings, an argument of the exponent rounded twice, which is worth z^2 exp(-z^2) < 0.4 roundings of it
# in all, and six operations on terms that are at most 1.2 (1 + |g|) of: less than 32 roundings of 1 + |g|.
GATE = 32 * U


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def i8(x, by_columns=False):
    """(codes, scales) of the rows (columns) of x, in 64 bits; a line that is not finite has scale NaN and codes 0."""
    x = (x.t() if by_columns else x).double()
    top = x.abs().amax(1)
    fine = torch.isfinite(top)
    scales = torch.where(fine, top, 0.0).float()
    scales = scales * (torch.ones_like(scales) / torch.full_like(scales, 127.0))
    t = torch.where(fine[:, None], x, 0.0) / torch.where(scales > 0, scales, 1.0).double()[:, None]
    t = torch.where(scales[:, None] > 0, t, 0.0)
    low = torch.floor(t)
    rest = t - low
    codes = (low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 != 0)))).clamp(-127, 127)
    return codes, torch.where(fine, scales, math.nan)


def padded_codes(codes):
    rows, cols = codes.shape
    wide = torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.int8, device=codes.device)
    wide[:, :cols] = codes.to(torch.int8)
    return wide.view(torch.uint8)


def gate(g, kind):
    if kind == GELU:
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    s, rest = torch.sigmoid(g), torch.sigmoid(-g)
    return (s, s * rest) if kind == SIGMOID else (g * s, s + g * s * rest)


def rounded(x):
    """A bf16 operand's values."""
    return x.to(BF16).double()


def product(a, b, bias=None):
    """a b^T + bias, and a bound of the error of fp32 sums in any order: each of K products passes through at most K + 1 roundings."""
    y, size = a @ b.t(), a.abs() @ b.abs().t()
    off = (a.shape[1] + 2) * U * size
    if bias is not None:
        y = y + bias.double()
        off = off + U * y.abs() + U * size
    return y, off


def i8_product(codes, scales, w_codes, w_scales, bias=None):
    """Exact sums; their conversion, two factors, and the bias round once each."""
    y = (codes @ w_codes.t()) * scales.double()[:, None] * w_scales.double()
    off = 4 * U * y.abs()
    if bias is not None:
        y = y + bias.double()
        off = off + U * y.abs()
    return y, off


def gated(g, off_g, u, off_u, kind):
    """{name: (value, bound of the fp32 error)} of H and its slopes."""
    value, slope = gate(g, kind)
    off_value = STEEPEST[kind] * off_g + GATE * (1 + g.abs())
    off_slope = CURVED[kind] * off_g + GATE * (1 + g.abs())
    return {"h": (value * u, off_value * (u.abs() + off_u) + value.abs() * off_u + 2 * U * (value * u).abs()),
            "slope_u": (value, off_value),
            "slope_g": (u * slope, off_slope * (u.abs() + off_u) + slope.abs() * off_u + 2 * U * (u * slope).abs())}


def close(got, want, off, what=""):
    """got within `off` and one rounding to its type of want; NaN and infinities where they are."""
    got, want = got.double(), (want if want.dtype == torch.float64 else want.double())
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), what + ": other places are finite"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": other places are NaN"
    far = ((got - want).abs() - off)[fine]
    assert far.numel() == 0 or not (far > 0).any(), f"{what}: {int((far > 0).sum())} of {far.numel()} off, by {far.max().item():.3g} over the bound"


def check(got, want, off, what=""):
    h = half_step(got.dtype)
    tiny = 2.0 ** -133 if got.dtype == BF16 else 2.0 ** -149
    close(got, want, off + h * (want.abs() + off) * (1 + h) + tiny, what)
