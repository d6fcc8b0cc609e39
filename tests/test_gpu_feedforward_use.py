"""The feed-forward module as callers use it: several streams."""
import pytest
import torch

from paper_2205_03494_amd import omc
from paper_2205_03494_amd.feedforward import FeedForward

pytestmark = pytest.mark.gpu


def frames(rows, seed, width=96):
    return torch.randn(rows, width, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


def test_passes_on_two_streams_share_no_workspace(monkeypatch):
    """One after the other here, so that nothing is raced for; what a pass writes must still be its own."""
    m, used, real = FeedForward(96, 260), [], omc.omc_mx4_linear
    monkeypatch.setattr(omc, "omc_mx4_linear", lambda *a: (used.append((len(streams_done), a[5])), real(*a))[1])
    streams_done, x = [], frames(200, 1)
    want = m.forward(x)
    used.clear()
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            out = m.forward(x)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        streams_done.append(s)
    spans = [[(w.data_ptr(), w.data_ptr() + w.numel()) for i, w in used if i == k and w.numel()] for k in (0, 1)]
    assert spans[0] and spans[1]
    assert all(a1 <= b0 or b1 <= a0 for a0, a1 in spans[0] for b0, b1 in spans[1])
