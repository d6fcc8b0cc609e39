"""How far a gate in fp32 may be from its value by the value itself, far out too: what the steps of its arithmetic round, in roundings of 2^-24.

    e = exp2(c g), c = -log2 e in fp32 (off by 0.224 roundings): a product, so that the exponent is off by 1.224 roundings of itself and e by 1.224 |g| of its own; exp2 itself by 2 (a last place)
    s = 1 / (1 + e): less than e's where g < 0 and 0.35 elsewhere, a sum, a reciprocal by 2:              1.224 max(-g, 0) + 6;   g s: 1 more
    1 - s = e s: e's, s' and a product:                                                                   2.448 |g| + 10;         s (1 - s): 3.7 |g| + 17
    P(g) = erfc(-g / sqrt 2) / 2 for g < 0, exp2(c g g / 2) q(t): two products in the exponent, 2.224 g^2 / 2 of e; exp2 by 2; t = 1 / (1 + 0.295 |g|) by 3, which are worth 2.8 times as much of t q(t); q is
    fitted to 4.5e-7 (7.5); Horner's scheme rounds 3.2 of q; two products:                                1.112 g^2 + 25;         g P: 1 more
    P for g > 0, 1 - P(-g): g^2 P(-g) is at most 0.17 and P at least a half:                              26;                     g P: 1 more

The squares of these are less than a hundredth of them."""
import math

import torch

import products_ref as ref


def exact(g, kind):
    """(act, act', sum of the magnitudes of what act' adds up)"""
    value, slope = ref.gate(g, kind)
    if kind == ref.SIGMOID:
        return value, slope, slope
    if kind == ref.SWISH:
        s, rest = torch.sigmoid(g), torch.sigmoid(-g)
        return value, slope, s + (g * s * rest).abs()
    return value, slope, 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + (g * torch.exp(-0.5 * g * g)).abs() / math.sqrt(2.0 * math.pi)


def bounds(g, kind):
    """Of act by itself, and of act' by its terms' magnitudes; relative."""
    if kind == ref.GELU:
        return (1.13 * g.clamp(max=0.0).square() + 28) * ref.U, (1.13 * g.square() + 32) * ref.U
    return (1.24 * (-g).clamp(min=0.0) + 7.2) * ref.U, (3.8 * g.abs() + 20) * ref.U


def arguments(kind, device="cpu"):
    """Down to where act and its terms are no less than 2^-120."""
    most = 12.5 if kind == ref.GELU else 83.0
    return torch.cat((torch.linspace(-most, most, 2001), torch.linspace(-6, 6, 1200), torch.linspace(-0.01, 0.01, 99))).to(device)


def check(g, h, slope_g, slope_u, kind):
    """h in any type and slopes (may be None) of act(g) * 1."""
    g = g.double()
    value, slope, terms = exact(g, kind)
    of_value, of_slope = bounds(g, kind)
    ref.check(h, value, of_value * value.abs(), "act")
    if slope_u is not None:
        ref.check(slope_u, value, of_value * value.abs(), "slope_u")
        ref.check(slope_g, slope, of_slope * terms, "slope_g")
