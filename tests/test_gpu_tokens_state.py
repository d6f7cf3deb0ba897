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


def test_backward_after_replay():
    """A forward in a graph, others in between, a replay: the backward that follows belongs to the replay."""
    net = network(T=12, every=True, norm=True, seed=8)
    net.forward(B_TH)
    g = pipeline.Graphed(lambda: net.forward(B_TH).readout_steps())
    for seed in range(3):
        between, X = (network(T=12, every=True, norm=True, seed=s).X for s in (30 + seed, 40 + seed))
        net.X.copy_(between)
        net.forward(B_TH)
        net.sparse_backward(net.compact(B_TH))
        net.X.copy_(X)
        ro = g()
        torch.cuda.synchronize()
        got = net.sparse_backward(net.compact(B_TH), ro)
        other = fresh(net, X)
        other.forward(B_TH)
        want = other.sparse_backward(other.compact(B_TH))
        assert torch.equal(got[1], want[1]) and all(torch.equal(p, q) for p, q in zip(got[0], want[0]))
        assert all(torch.equal(p, q) for p, q in zip(net.norm_grads, other.norm_grads))


def test_norm_gradients_of_a_replay():
    """norm_grads after a captured backward's replay, an eager one in between; a step's own gradients stay as they were."""
    net = network(T=12, every=True, norm=True, seed=9)
    net.forward(B_TH)
    csrs = net.compact(B_TH)
    net.sparse_backward(csrs)
    want = [t.clone() for t in net.norm_grads]
    ro = net.readout_steps()
    g = pipeline.Graphed(lambda: net.sparse_backward(csrs, ro))
    for _ in range(3):
        net.sparse_backward(csrs, (2.0 * ro[0], ro[1], ro[2]))
        assert all(torch.equal(2.0 * p, q) for p, q in zip(want, net.norm_grads))
        g()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, net.norm_grads))
    opt = pipeline.Adam(net.params(), lr=1e-3)
    one = net.train_step(opt, B_TH)["grads"]
    kept = [t.clone() for t in one]
    two = net.train_step(opt, B_TH)["grads"]
    assert all(torch.equal(p, q) for p, q in zip(one, kept)) and not torch.equal(one[-1], two[-1])
