"""Gradients of a gated layer against differences of its forward pass, along directions in which the difference does not cancel.

A direction is the sign of a gradient in 64 bits, so that the difference of sum(R H) is the sum of all its magnitudes, and a gradient that lacks a term lies far from it.  Steps are held by bf16: operands
are whole multiples of their steps, at most 255 of them, so that X +- e D has no rounding."""
import torch

import products_ref as ref

F64 = torch.float64
NAMES = ("X", "Wg", "Wu", "bg", "bu")
THIRD = 1.6                          # |act''| and |act'''| are at most this
POWER = 10                           # so many times its bound has a difference to be, to tell anything


class Layer:
    """Operands on `device`, and the layer's terms in 64 bits."""

    def __init__(self, M, N, K, kind, seed, device):
        gen = torch.Generator(device).manual_seed(seed)

        def grid(rows, cols, step):
            return (torch.randint(-96, 97, (rows, cols), device=device, generator=gen).float() * step).to(ref.BF16)
        self.kind, self.M, self.N, self.K, self.device = kind, M, N, K, device
        self.steps = {"X": 2.0 ** -9, "Wg": 2.0 ** -6, "Wu": 2.0 ** -6, "bg": 2.0 ** -6, "bu": 2.0 ** -6}
        self.at = {"X": grid(M, K, self.steps["X"]), "Wg": grid(N, K, self.steps["Wg"]), "Wu": grid(N, K, self.steps["Wu"]),
                   "bg": torch.randn(N, device=device, generator=gen), "bu": torch.randn(N, device=device, generator=gen)}
        x, wg, wu, bg, bu = (self.at[n].double() for n in NAMES)
        self.g, self.u = x @ wg.t() + bg, x @ wu.t() + bu
        self.value, self.slope = ref.gate(self.g, kind)
        # dH: of one sign with a column's terms of dg in half of the columns, with those of du in the others, so that long columns' sums do not cancel
        sign = torch.where(torch.arange(N, device=device) % 2 == 0, torch.sign(self.u * self.slope), torch.sign(self.value)).float()
        self.R = torch.randn(M, N, device=device, generator=gen).abs() * sign

    def gradients(self, without=None):
        """In 64 bits; `without` dg or du, one of X's two terms."""
        x, wg, wu, _, _ = (self.at[n].double() for n in NAMES)
        dg, du = self.R.double() * self.u * self.slope, self.R.double() * self.value
        dx = (0 if without == "dg" else dg @ wg) + (0 if without == "du" else du @ wu)
        return {"X": dx, "Wg": dg.t() @ x, "Wu": du.t() @ x, "bg": dg.sum(0), "bu": du.sum(0)}

    def directions(self):
        return {n: torch.where(t < 0, -1.0, 1.0).to(self.device) for n, t in self.gradients().items()}

    def moved(self, name, direction, sign):
        """All operands, `name` a step away."""
        operands = dict(self.at)
        t = operands[name]
        there = t.float() + sign * self.steps[name] * direction.float()
        operands[name] = there.to(t.dtype)
        assert t.dtype != ref.BF16 or torch.equal(operands[name].float(), there)
        return [operands[n] for n in NAMES]

    def bound(self, name, direction):
        """Of what may lie between the difference of sum(R H), H in fp32, and the product of the direction with gradients of bf16 slopes: each slope is rounded once, and dg and du once more for the products
        (2^-8 of every term, or twice that; the squares are a hundredth of it); the difference's own third-order term; sums of fp32, in H twice."""
        x, wg, wu, bg, bu = (self.at[n].double() for n in NAMES)
        r, e, d, zero = self.R.double().abs(), self.steps[name], direction.double(), torch.zeros_like(self.g)
        if name == "X":
            step_g, step_u, sum_g, sum_u = d @ wg.t(), d @ wu.t(), wg.abs().sum(1), wu.abs().sum(1)
        else:
            step = d.expand_as(zero) if name[0] == "b" else x @ d.t()
            size = 1 if name[0] == "b" else x.abs().sum(1, keepdim=True)
            step_g, step_u, sum_g, sum_u = (step, zero, size, 0) if name[1] == "g" else (zero, step, 0, size)
        a, b = e * step_g.abs(), e * step_u.abs()
        terms = (r * ((self.u * self.slope).abs() * a + self.value.abs() * b)).sum()
        third = (r * THIRD * (a ** 3 * (self.u.abs() + b) + 3 * a ** 2 * b)).sum() / 6
        size_g, size_u = x.abs() @ wg.abs().t() + bg.abs(), x.abs() @ wu.abs().t() + bu.abs()
        sums = (self.K + 8) * ref.U * (r * (1.2 * size_g * self.u.abs() + self.value.abs() * size_u + 8 * (1 + self.g.abs()) * self.u.abs())).sum()
        # and the gradient's own sums, of at most 2 N or M terms
        own = (max(self.M, 2 * self.N) + 2) * ref.U * e * (r * ((self.u * self.slope).abs() * sum_g + self.value.abs() * sum_u)).sum()
        return ((2.02 if name[0] in "XW" else 1.01) * 2.0 ** -8 * terms + third + sums + own).item()

    def compare(self, name, gradient, direction, plus, minus):
        """plus and minus: sum(R H) a step ahead and a step behind."""
        difference, bound = (plus - minus) / 2, self.bound(name, direction)
        product = self.steps[name] * (gradient.double() * direction.double()).sum().item()
        assert abs(difference) >= POWER * bound, (name, "tells nothing", difference, bound)
        assert abs(product - difference) <= bound, (name, product, difference, bound)

    def objective(self, X, Wg, Wu, bg, bu):
        """sum(R H) in 64 bits."""
        g, u = X.double() @ Wg.double().t() + bg.double(), X.double() @ Wu.double().t() + bu.double()
        return (self.R.double() * ref.gate(g, self.kind)[0] * u).sum().item()
