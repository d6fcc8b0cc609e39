"""I8's scale is the product a * (1 / 127) in fp32 and not the quotient a / 127: where they differ, codes differ too, so that only one of them can be the format's."""
import torch

import products_ref as ref

BF16 = torch.bfloat16


def halves(exponents=(-104, -3, 0, 5, 100)):
    """Rows of [a, a / 2, -a / 2, 0] with a of every bf16 significand."""
    a = torch.cat([(1.0 + torch.arange(128) / 128.0) * 2.0 ** e for e in exponents])
    x = torch.stack((a, a / 2, -a / 2, torch.zeros_like(a)), 1)
    assert torch.equal(x.to(BF16).float(), x)
    return x


def quotients(x):
    """Codes by the rounded quotient."""
    scales = (x.double().abs().amax(1) / 127.0).float()
    return torch.round(x.double() / scales.double()[:, None]), scales


def test_the_references_scale_is_the_product():
    x = halves((0,))
    a = x[:, 0]
    codes, scales = ref.i8(x)
    assert torch.equal(scales, a * torch.tensor(1.0 / 127.0, dtype=torch.float32))
    other_codes, other = quotients(x)
    differ = scales != other
    assert differ.sum() == 6
    # half the largest magnitude is 63.5 by either, but for the scale's rounding
    assert torch.equal((codes != other_codes).any(1), differ)
    assert (codes[:, 0] == 127).all() and (other_codes[:, 0] == 127).all()


def test_bf16_values_are_rounded_once():
    """s times a code in fp32 and then in bf16 is the exact product in bf16, for every significand of a largest magnitude in bf16 and every code."""
    scales = (1.0 + torch.arange(128) / 128.0) * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    codes = torch.arange(1, 128)
    twice = (scales[:, None] * codes.float()).to(BF16).double()
    significand, exponent = torch.frexp(scales.double()[:, None] * codes.double())
    assert torch.equal(twice, torch.ldexp(torch.round(significand * 256), exponent - 8))


def test_a_scale_below_the_quotient_still_gives_127():
    """Codes saturate only where scales are subnormal."""
    g = torch.Generator().manual_seed(1)
    a = torch.rand(200000, generator=g) + 1.0
    scales = a * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    assert (scales.double() < a.double() / 127.0).any()
    assert (torch.round(a.double() / scales.double()) == 127).all()
    tiny = torch.tensor([[2.0 ** -149 * 190, 0.0]])
    assert 190 / round(190 / 127) > 127.5 and ref.i8(tiny)[0][0, 0] == 127
