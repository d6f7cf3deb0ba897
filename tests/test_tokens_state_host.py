"""Networks on tokens: answers and gradients belong to the device's present state, not to the last Python call. The
library's calls are replaced by recorders, so that this runs without a device."""
import pytest
import torch

from paper_2105_08810_amd import pipeline, snn


def network(T=4, B=3, V=7, N=5, C=2, norm=False):
    n = pipeline.Norm(torch.ones(N), torch.zeros(N)) if norm else None
    return pipeline.Network(X=torch.zeros((T, B), dtype=torch.int32), Ws=[torch.zeros((V, N))], W_out=torch.zeros((N, C)),
                            alphas=[0.9], alpha_out=0.9, labels=torch.zeros((T, B), dtype=torch.int32), loss_mode=1, norm_in=n)


def test_membrane_is_formed_at_each_call(monkeypatch):
    """What a graph's replay or an optimizer changes shows in the next call."""
    calls = []

    def forward(s_in, W, T, B, N_in, N_out, alpha, theta, V, S, trace=None):
        calls.append(1)
        V.fill_(float(s_in.sum()) + 100 * float(W.sum()))

    monkeypatch.setattr(snn, "snn_lif_forward", forward)
    net = network()
    net.allocate()
    net.S[-1].zero_()
    first = net.membrane()
    assert not first.any()
    net.S[-1][0, 0, 0] = 3  # as a replay does
    assert bool((net.membrane() == 3).all())
    net.W_out[0, 0] = 1.0  # as an optimizer's step does
    assert bool((net.membrane() == 103).all())
    assert not first.any() and len(calls) == 3


def test_norm_state_is_in_buffers(monkeypatch):
    """The norm's means and deviations, and its gradients, are where a replay of an earlier capture writes them: the same
    tensors in every forward and backward."""
    seen = {"forward": [], "backward": []}
    monkeypatch.setattr(snn, "embed", lambda *a, out=None, **k: out)
    monkeypatch.setattr(snn, "layer_norm", lambda x, *a, out=None, **k: seen["forward"].append(
        (torch.empty(x.shape[:-1]), torch.empty(x.shape[:-1]))) or (out, *seen["forward"][-1]))
    monkeypatch.setattr(snn, "snn_layer_norm", lambda x, g, b, e, y, mean, rstd, **k: seen["forward"].append((mean, rstd)))
    monkeypatch.setattr(snn, "snn_lif_forward_currents", lambda *a, **k: None)
    net = network(norm=True)
    net.forward()
    net.forward()
    for mean, rstd in seen["forward"]:
        assert mean.data_ptr() == seen["forward"][0][0].data_ptr() and rstd.data_ptr() == seen["forward"][0][1].data_ptr()

    def grad(dy, x, gamma, mean, rstd, *a, **k):
        seen["backward"].append((mean.data_ptr(), rstd.data_ptr()))
        return torch.empty_like(x), torch.empty(5), torch.empty(5)

    monkeypatch.setattr(snn, "leak_grad", lambda eps, alpha, shape, **k: torch.zeros(shape))
    monkeypatch.setattr(snn, "layer_norm_grad", grad)
    monkeypatch.setattr(snn, "snn_layer_norm_grad", grad)
    monkeypatch.setattr(snn, "snn_layer_norm_grad_workspace", lambda *a: 1)
    monkeypatch.setattr(snn, "embed_grad", lambda ids, d, V, scale: torch.zeros((V, d.shape[-1])))
    net._backward_tokens(None, None)
    first = [g.data_ptr() for g in net.norm_grads]
    keep = net.norm_grads  # its memory is not handed out again
    net._backward_tokens(None, None)
    assert [g.data_ptr() for g in net.norm_grads] == first and keep is not None
    assert all(p == tuple(t.data_ptr() for t in seen["forward"][0]) for p in seen["backward"])
