"""Networks on tokens under captured graphs and optimizer steps between the calls: answers and gradients are those of the
state that the device holds."""
import copy

import pytest
import torch

from paper_2105_08810_amd import pipeline
from test_gpu_tokens_pipeline import B_TH, network

pytestmark = pytest.mark.gpu


def fresh(net, X):
    """The same weights on X, in a network of its own."""
    other = copy.copy(net)
    other.X, other.V, other.S, other.bits = X.clone(), [], [], []
    return other


def test_answers_between_replays():
    """membrane(), record() and draw() after a replay on new tokens, and after W_out has changed."""
    net = network(T=12, every=True, norm=True, seed=8)
    net.forward(B_TH)
    g = pipeline.Graphed(lambda: net.forward(B_TH).readout_steps())
    u = torch.linspace(0.05, 0.95, net.T * net.B, device="cuda").view(net.T, net.B)
    seen = []
    for seed in range(4):
        X = network(T=12, every=True, norm=True, seed=20 + seed).X
        net.X.copy_(X)
        g()
        torch.cuda.synchronize()
        other = fresh(net, X)
        other.forward(B_TH)
        want = other.membrane()
        assert torch.equal(net.membrane(), want)
        assert all(torch.equal(p, q) for p, q in zip(net.draw(u), other.draw(u)))
        assert torch.equal(net.draw(u[3], step=3)[0], other.draw(u)[0][3])
        a, b = net.record(3), other.record(3)
        assert torch.equal(a.ids, b.ids) and torch.equal(a.vals, b.vals) and torch.equal(a.lse, b.lse)
        seen.append(want)
        net.W_out.mul_(1.25)
        other.W_out = net.W_out
        assert torch.equal(net.membrane(), other.membrane()) and not torch.equal(net.membrane(), want)
    assert not torch.equal(seen[0], seen[1])
