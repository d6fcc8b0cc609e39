"""The comparison of gradients with differences tells: right gradients pass, and wrong ones do not, at every size that the kernels are compared at."""
import pytest
import torch

import differences_ref as differences
import products_ref as ref
from test_gpu_products_differences import SIZES


def rounded(layer):
    """The layer's gradients as its backward pass defines them: bf16 slopes, dg and du in bf16 for the products."""
    x, wg, wu = (layer.at[n].double() for n in ("X", "Wg", "Wu"))
    dg, du = (layer.R * ref.rounded(s).float() for s in (layer.u * layer.slope, layer.value))
    rg, ru = ref.rounded(dg), ref.rounded(du)
    return {"X": rg @ wg + ru @ wu, "Wg": rg.t() @ x, "Wu": ru.t() @ x, "bg": dg.double().sum(0), "bu": du.double().sum(0)}


@pytest.mark.parametrize("kind", (ref.SIGMOID, ref.SWISH, ref.GELU))
@pytest.mark.parametrize("size", SIZES)
def test_wrong_gradients_are_told(size, kind):
    layer = differences.Layer(*size, kind, 30, "cpu")
    directions, right = layer.directions(), rounded(layer)
    other = {"Wg": "Wu", "Wu": "Wg", "bg": "bu", "bu": "bg"}
    for name in differences.NAMES:
        plus, minus = (layer.objective(*layer.moved(name, directions[name], s)) for s in (1, -1))
        layer.compare(name, right[name], directions[name], plus, minus)
        wrong = [torch.zeros_like(right[name]), -right[name], 0.9 * right[name], 1.1 * right[name]]
        if name == "X":
            wrong += [layer.gradients("dg")["X"], layer.gradients("du")["X"]]
        else:
            wrong += [right[other[name]]]
        for i, w in enumerate(wrong):
            with pytest.raises(AssertionError):
                layer.compare(name, w, directions[name], plus, minus)
                pytest.fail(f"{name}: {i} passes")


def test_directions_that_cancel_are_refused():
    layer = differences.Layer(96, 72, 64, ref.SWISH, 30, "cpu")
    gradient = layer.gradients()["bg"]
    in_turn = torch.where(gradient.abs().argsort().argsort() % 2 == 0, 1.0, -1.0) * torch.sign(gradient).float()    # by size, once ahead and once behind
    plus, minus = (layer.objective(*layer.moved("bg", in_turn, s)) for s in (1, -1))
    with pytest.raises(AssertionError, match="tells nothing"):
        layer.compare("bg", gradient, in_turn, plus, minus)
