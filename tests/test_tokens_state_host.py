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


def test_one_step_of_a_large_vocabulary(monkeypatch):
    """One step's rows are formed for slices of the samples; all steps together are refused where they cannot be."""
    formed = []

    def forward(s_in, W, T, B, N_in, N_out, alpha, theta, V, S, trace=None):
        formed.append((T, B, N_out))
        assert s_in.is_contiguous() and s_in.shape == (T, B, N_in) and V.shape == S.shape == (T, B, N_out)
        V[-1] = s_in[-1, :, :1].float()

    monkeypatch.setattr(snn, "snn_lif_forward", forward)
    net = network(T=6, B=5)
    net.allocate()
    net.S[-1].copy_(torch.arange(6 * 5).view(6, 5, 1).expand(6, 5, 5))
    assert torch.equal(net.membrane(3), torch.arange(15.0, 20.0)[:, None].expand(5, 2)) and formed == [(4, 5, 2)]
    formed.clear()
    monkeypatch.setattr(pipeline.Network, "kSliceValues", 17)  # two samples of 4 x 2 values
    assert torch.equal(net.membrane(3), torch.arange(15.0, 20.0)[:, None].expand(5, 2))
    assert formed == [(4, 2, 2), (4, 2, 2), (4, 1, 2)]
    formed.clear()
    monkeypatch.setattr(pipeline.Network, "kSliceValues", 1)  # never less than a sample
    assert torch.equal(net.membrane(-1), torch.arange(25.0, 30.0)[:, None].expand(5, 2)) and formed == [(6, 1, 2)] * 5
    formed.clear()
    monkeypatch.setattr(pipeline.Network, "kClasses", 3)  # classes by slices too
    net.W_out = torch.zeros((5, 8))
    monkeypatch.setattr(pipeline.Network, "kSliceValues", 48)  # four samples of 4 x 3 values
    assert torch.equal(net.membrane(3), torch.arange(15.0, 20.0)[:, None].expand(5, 8))
    assert formed == [(4, 4, 3), (4, 1, 3), (4, 4, 3), (4, 1, 3), (4, 4, 2), (4, 1, 2)]
    formed.clear()
    assert torch.equal(net.membrane()[-1], torch.arange(25.0, 30.0)[:, None].expand(5, 8))
    assert formed == [(6, 5, 3), (6, 5, 3), (6, 5, 2)]
    for step in (6, -7):
        with pytest.raises(IndexError):
            net.membrane(step)
    net.W_out = torch.empty((5, 1), device="meta").expand(5, 1 << 27)
    formed.clear()
    with pytest.raises(ValueError, match="name a step"):
        net.membrane()
    with pytest.raises(ValueError, match="name a step"):
        net.record(3)
    assert not formed


@pytest.mark.parametrize("eps", [0.0, -1e-5, float("inf"), float("nan")])
def test_norm_needs_eps(eps):
    """With eps 0 a padded step's currents would be NaN."""
    with pytest.raises(ValueError, match="eps"):
        pipeline.Network(X=torch.zeros((4, 3), dtype=torch.int32), Ws=[torch.zeros((7, 5))], W_out=torch.zeros((5, 2)),
                         alphas=[0.9], alpha_out=0.9, labels=torch.zeros((4, 3), dtype=torch.int32), loss_mode=1,
                         norm_in=pipeline.Norm(torch.ones(5), torch.zeros(5), eps))


def test_each_kind_has_its_readout():
    """A readout of the other kind of target is refused before any device call."""
    net = network()
    net.allocate()
    with pytest.raises(ValueError, match="every step"):
        net.readout_distilled(pipeline.Distill(pipeline.Record(None, None, None)))
    net.labels = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="readout\\(\\)"):
        net.readout_steps()
