"""The layer's operators as a module uses them: forward, backward and update of a feed-forward module, and single frames."""
import numpy as np
import pytest
import torch

import mx4_ref as ref
from paper_2205_03494_amd import omc
from paper_2205_03494_amd.feedforward import EPS, FeedForward

pytestmark = pytest.mark.gpu


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def bf16(a):
    return torch.from_numpy(a).to(torch.bfloat16).double().numpy()


def close(got, want, share):
    """By the 2-norm: a value that lies on the edge of a rounding may fall to its other side."""
    got = ref.as64(got)
    assert np.linalg.norm(got - want) <= share * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("frames", [1, 7, 48, 200])
def test_module_against_the_same_in_64_bits(frames):
    d, f = 96, 260
    m = FeedForward(d, f, seed=3)
    g = torch.Generator("cuda").manual_seed(frames)
    x, dout = torch.randn(frames, d, device="cuda", generator=g), torch.randn(frames, d, device="cuda", generator=g)
    out = m.forward(x, keep=True)
    dx = m.backward(dout)
    v = {n: ref.as64(m.value(n)) for n in m.shapes}
    q = lambda a: ref.quantize(a)[2]
    x64, do = ref.as64(x), ref.as64(dout)
    y, mean, rstd = ref.layer_norm(x64, v["gamma"], v["beta"], EPS)
    y = bf16(y)
    h = bf16(q(y) @ q(v["w1"].T).T + v["b1"])
    a = bf16(h * bf16(sigmoid(h)))
    z = q(a) @ q(v["w2"].T).T + v["b2"]
    # bf16 activations are rounded twice on their way (2^-9 of each), and a rounding to 4 bits that goes the other way moves one value by a step: a few in ten thousand
    close(out, x64 + 0.5 * z, 0.01)
    dz = bf16(0.5 * do)
    da = bf16(q(dz) @ q(v["w2"]).T)
    close(m.grad("w2"), q(a.T) @ q(dz.T).T, 0.02)
    close(m.grad("b2"), dz.sum(0), 1e-5)
    s = sigmoid(h)
    dh = bf16(da * s * (1 + h * (1 - s)))
    dy = bf16(q(dh) @ q(v["w1"]).T)
    close(m.grad("w1"), q(y.T) @ q(dh.T).T, 0.03)
    close(m.grad("b1"), dh.sum(0), 0.02)
    want = ref.layer_norm_backward(dy, x64, v["gamma"], mean, rstd)
    close(dx, want[0] + do, 0.01)
    close(m.grad("gamma"), want[1], 0.03)
    close(m.grad("beta"), want[2], 0.03)


@pytest.mark.parametrize("kind", [omc.OMC_SGD, omc.OMC_MOMENTUM, omc.OMC_ADAM])
def test_training_lowers_the_loss(kind):
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(256, 128, device="cuda", generator=g)
    target = x + 0.3 * torch.tanh(x.roll(1, 1))
    m, losses = FeedForward(128, 512), []
    for t in range(1, 16):
        diff = m.forward(x, keep=True) - target
        losses.append(diff.square().mean().item())
        m.backward(diff * (2.0 / diff.numel()))
        m.step(omc.opt(kind, {omc.OMC_SGD: 5.0, omc.OMC_MOMENTUM: 1.0, omc.OMC_ADAM: 2e-3}[kind], t=t))
    assert losses[-1] < 0.7 * losses[0]


def test_frames_one_by_one_are_the_batch():
    """Rows are rounded each for itself; only the order of the products' sums differs, which may take an activation over the edge of a rounding to 4 bits: by 0.5 at most here, half a
    row of W2 (norm 0.5), against an output of norm 22."""
    m = FeedForward(512, 2048)
    x = torch.randn(70, 512, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    batch = m.forward(x)
    for i in (0, 33, 69):
        close(m.forward(x[i:i + 1]), ref.as64(batch[i:i + 1]), 0.01)
