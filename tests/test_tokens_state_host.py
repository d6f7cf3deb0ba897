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
