"""Networks on tokens under captured graphs and optimizer steps between the calls: answers and gradients are those of the
state that the device holds."""
import copy

import pytest
import torch

from paper_2105_08810_amd import pipeline, snn
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


@pytest.mark.parametrize("per", [1, 3, 1 << 28])
def test_one_step_by_slices(per, monkeypatch):
    """One step's rows are those of the whole membrane, to the bit, however many samples are formed together."""
    net = network(T=30, B=7, every=True, seed=11, sizes=(64, 48), C=130)
    net.forward()
    want = net.membrane()
    u = torch.linspace(0.05, 0.95, 7, device="cuda")
    for step in (0, 1, 17, 29, -1):
        monkeypatch.setattr(pipeline.Network, "kSliceValues", per * 130 * (step % 30 + 1))
        assert torch.equal(net.membrane(step), want[step])
        assert all(torch.equal(p, q) for p, q in zip(net.draw(u, step=step), snn.readout_sample(want[step], u)))


def test_more_classes_than_one_forward_takes():
    """5000 classes: the membrane is that of either half of them, and records and draws read it."""
    net = network(T=15, B=4, every=True, seed=13, C=5000)
    net.forward()
    V = net.membrane()
    half = copy.copy(net)
    for c in (slice(0, 2500), slice(2500, 5000)):
        half.W_out = net.W_out[:, c].contiguous()
        assert torch.equal(half.membrane(), V[..., c])
    assert torch.equal(net.membrane(9), V[9])
    rec = net.record(3)
    assert torch.equal(rec.vals[..., 0], V.amax(2))
    cls, _, _ = net.draw(torch.full((15, 4), 0.5, device="cuda"), torch.zeros((15, 4), device="cuda"))
    assert torch.equal(V.gather(2, cls.long()[..., None])[..., 0], V.amax(2))


def test_draw_over_a_large_vocabulary():
    """A step of 500 x 256 samples over 32003 classes, whose membrane would have 4.1e9 values."""
    net = network(T=500, B=256, V=50, sizes=(64,), C=32003, every=True, seed=12)
    net.forward()
    cls, logp, _ = net.draw(torch.full((256,), 0.5, device="cuda"), torch.zeros(256, device="cuda"), step=250)
    z = net.trace_out[250].double() @ net.W_out.double()
    best = z.max(1)
    # the membrane is a sum of 250 steps of at most 64 spikes' rows, each rounded: 2^-24 of its absolute sum a step
    tol = 500 * 2.0 ** -24 * float((net.trace_out[250].double() @ net.W_out.double().abs()).max())
    assert bool((z.gather(1, cls.long()[:, None])[:, 0] >= best.values - 2 * tol).all())
    assert bool(torch.isfinite(logp).all())
    with pytest.raises(ValueError, match="name a step"):
        net.draw(torch.zeros((500, 256), device="cuda"))


def test_tokens_outside_the_vocabulary():
    """Without a norm they are no spike; behind it their current is beta."""
    for norm in (False, True):
        net = network(T=10, every=True, norm=norm, seed=14)
        net.X.fill_(-1)
        net.X[4, 2] = 10 ** 6
        out = net.train_step(pipeline.Adam(net.params(), lr=1e-3), B_TH)
        assert not bool(out["grads"][0].any())
        net = network(T=10, every=True, norm=norm, seed=14)
        net.X.fill_(-1)
        net.forward()
        V, S = net.V[0], net.S[0].float()
        for t in range(9):
            current = net.norm_in.beta.double() if norm else 0.0
            want = 0.9 * V[t].double() + current - S[t].double()
            assert float((V[t + 1].double() - want).abs().max()) < 4 * 2.0 ** -24 * (1 + float(V.abs().max()))
