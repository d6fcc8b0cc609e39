"""The bounds of the gates by their own values: the arithmetic that they are derived from keeps them, and what loses a tail does not."""
import math

import numpy as np
import pytest
import torch

import products_ref as ref
import tails_ref as tails

KINDS = (ref.SIGMOID, ref.SWISH, ref.GELU)


def exact(kind):
    g = tails.arguments(kind)
    value, slope, _ = tails.exact(g.double(), kind)
    return g, value, slope


@pytest.mark.parametrize("kind", KINDS)
def test_rounded_exact_values_pass(kind):
    g, value, slope = exact(kind)
    tails.check(g, value.float(), slope.to(ref.BF16), value.to(ref.BF16), kind)
    assert value.abs()[g != 0].min() > 2.0 ** -122


@pytest.mark.parametrize("kind", (ref.SIGMOID, ref.SWISH))
def test_exponentials_in_fp32_with_errors_of_a_last_place_pass(kind):
    g = tails.arguments(kind)
    for way in (-1.0, 0.0, 1.0):                       # exp2 and reciprocal a last place to either side
        off = 1.0 + way * 2.0 ** -23
        e = (torch.exp2((g * torch.tensor(-1.44269504088896340736)).double()) * off).float()
        s = (off / (1.0 + e).double()).float()
        rest = e * s
        value = s if kind == ref.SIGMOID else g * s
        slope = s * rest if kind == ref.SIGMOID else value * rest + s
        tails.check(g, value, slope.to(ref.BF16), value.to(ref.BF16), kind)


@pytest.mark.parametrize("kind", KINDS)
def test_lost_tails_do_not(kind):
    g, value, slope = exact(kind)
    far = g < -4.0
    lost = {"nothing": torch.where(far, 0.0, value), "a part in a thousand": torch.where(far, value * 1.001, value), "the neighbour's": torch.where(far, value.roll(1), value)}
    wide = g.double()
    if kind == ref.GELU:
        lost["a difference"] = (0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))).double()
        lost["tanh"] = 0.5 * wide * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (wide + 0.044715 * wide ** 3)))
    else:
        lost["half a tanh"] = ((0.5 + 0.5 * torch.tanh(0.5 * g)) * (1.0 if kind == ref.SIGMOID else g)).double()
    for name, h in lost.items():
        with pytest.raises(AssertionError, match="act"):
            tails.check(g, h.float(), None, None, kind)
    for name, wrong in (("nothing", torch.where(far, 0.0, slope)), ("a hundredth", slope * 1.01), ("another sign", -slope)):
        with pytest.raises(AssertionError, match="slope_g"):
            tails.check(g, value.float(), wrong.to(ref.BF16), value.to(ref.BF16), kind)


def test_the_old_bound_is_absolute():
    """Why these are beside it: the bound of products_ref.gated lets a gate that is nothing at -14 pass."""
    g = torch.tensor([-14.0], dtype=torch.float64)
    for kind in KINDS:
        want, off = ref.gated(g, 0 * g, 1 + 0 * g, 0 * g, kind)["h"]
        ref.check(torch.zeros(1), want, off)


def test_every_fp32_number_near_the_ends_is_normal():
    for kind in KINDS:
        _, slope, terms = tails.exact(tails.arguments(kind).double(), kind)
        assert terms.min() > 2.0 ** -122 and np.isfinite(slope.numpy()).all()
