"""Networks with the readout's row operators: a record of a forward, training steps with a distillation term (sparse and
dense, both loss modes, both kinds of network), drawing, and the example that runs them together."""
import math
import os
import sys

import numpy as np
import pytest
import torch

from oracle import rows
from paper_2105_08810_amd import pipeline, snn
from synth import CONFIGS, make_inputs

pytestmark = pytest.mark.gpu


def _net(mode, seed=0):
    net = pipeline.from_inputs(make_inputs(CONFIGS["tiny"]))
    net.loss_mode = mode
    g = torch.Generator(device="cuda").manual_seed(seed)
    net.W_out = torch.randn(net.W_out.shape, generator=g, device="cuda")
    return net


def _teacher(net, K, tau, lse=True):
    other = _net(net.loss_mode, seed=7)
    rec = other.forward().record(K, tau)
    return rec if lse else pipeline.Record(rec.ids, rec.vals, None, tau)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("lse", [False, True])
def test_readout_distilled(mode, dense, lse):
    net = _net(mode).forward(0.2)
    T, B, C = net.V_out.shape
    rec = _teacher(net, 2, 1.5, lse)
    w = torch.rand((T, B), device="cuda")
    w[:3] = 0.0
    plain = net.readout(dense=True)
    csr, eps, ce, eps_dense, kd = net.readout_distilled(pipeline.Distill(rec, w), dense)
    z = net.V_out.view(T * B, C).cpu().numpy()
    cpu = lambda t: None if t is None else t.reshape(T * B, -1).squeeze(-1).cpu().numpy() if t.dim() == 2 else t.reshape(T * B, -1).cpu().numpy()  # noqa: E731
    loss, _, g, env, _ = rows.distill(z, cpu(rec.ids), cpu(rec.vals), cpu(rec.lse), 1.5, w.view(-1).cpu().numpy())
    want = plain[3].view(T * B, C).cpu().numpy() + g
    got = eps.view(T * B, C).cpu().numpy()
    # roundings of the distillation's gradient (its terms env) and of one addition
    assert (np.abs(got - want) <= 2.0 ** -24 * (200 * env + 2 * np.abs(want)) + 2.0 ** -24).all()
    assert abs(float(kd) - loss) <= 1e-5 * max(1.0, abs(loss))
    assert torch.equal(ce, plain[2])
    assert csr.row_ptr.cpu().tolist() == list(range(0, T * B * C + 1, C))
    assert csr.col_idx[:T * B * C].view(-1, C).cpu().tolist() == [list(range(C))] * (T * B)
    assert (eps_dense is not None) == dense
    if dense:
        assert torch.equal(eps_dense.view(-1), eps.view(-1))


@pytest.mark.parametrize("mode", [0, 1])
def test_training_step_with_distillation(mode):
    """The sparse and the dense step give the same readout gradient, which is the losses' difference along a direction
    (the losses are smooth in W_out away from ties of the maximum over time)."""
    distill = lambda net: pipeline.Distill(_teacher(net, 2, 1.5), scale=3.0)  # noqa: E731
    grads, out = {}, {}
    for sparse in (True, False):
        net = _net(mode)
        opt = pipeline.Adam(net.params(), lr=0.0)
        out[sparse] = net.train_step(opt, 0.2, sparse=sparse, distill=distill(net))
        grads[sparse] = out[sparse]["grads"]
    assert float(out[True]["kd"]) == float(out[False]["kd"]) and float(out[True]["kd"]) > 0
    for a, b in zip(grads[True], grads[False]):
        scale = float(b.abs().max())
        assert float((a - b).abs().max()) <= 1e-4 * scale + 1e-7
    net = _net(mode)
    W = net.W_out.clone()
    d = torch.randn(W.shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    d /= d.norm()
    h = 2e-3

    def total(x):
        net.W_out = x
        net.forward()
        ro = net.readout_distilled(distill(net))
        return float(ro[2]) + float(ro[4])

    diff = (total(W + h * d) - total(W - h * d)) / (2 * h)
    slope = float((grads[True][-1].double() * d.double()).sum())
    # float32 losses of size below 10, each within 1e-6 of themselves; curvature of traces of size below 10
    assert abs(diff - slope) <= 1e-5 / h + 0.02 * abs(slope) + 1e-3


def test_conv_training_step_with_distillation():
    """The conv network's sparse and dense steps agree on the gradients of cross-entropy and distillation."""
    inp = make_inputs(CONFIGS["conv"], list(range(2)))
    dev = torch.device("cuda")
    T, B = 12, 2
    X = torch.from_numpy(inp.X).to(dev)[:T].reshape(T, B, 28, 28, 1).contiguous()
    out = {}
    for sparse in (True, False):
        g = torch.Generator(device="cuda").manual_seed(0)
        net = pipeline.ConvNetwork(X=X, Wc=torch.randn((3, 3, 1, 8), generator=g, device=dev),
                                   W_out=torch.randn((14 * 14 * 8, 10), generator=g, device=dev) * 0.05, alpha=0.9,
                                   alpha_out=0.9, labels=torch.from_numpy(inp.labels.astype("int32")).to(dev), loss_mode=0)
        vals, ids = torch.randn((T, B, 10), generator=g, device=dev).topk(3, dim=2)
        rec = pipeline.Record(ids.to(torch.int32).contiguous(), vals.contiguous(), None, 1.0)
        out[sparse] = net.train_step(pipeline.Adam(net.params(), lr=0.0), 0.5, sparse=sparse,
                                     distill=pipeline.Distill(rec))
    assert float(out[True]["kd"]) == float(out[False]["kd"]) > 0
    for a, b in zip(out[True]["grads"], out[False]["grads"]):
        assert float((a - b).abs().max()) <= 1e-4 * float(b.abs().max()) + 1e-7


def test_step_without_distillation_is_unchanged():
    a, b = _net(0), _net(0)
    out = a.train_step(pipeline.Adam(a.params(), lr=0.0), 0.2)
    assert "kd" not in out
    b.forward(0.2)
    ro = b.readout()
    dWs, dW_out, _ = b.sparse_backward(b.compact(0.2), ro)
    assert torch.equal(out["grads"][0], dWs[0]) and torch.equal(out["grads"][1], dW_out)


def test_draw():
    net = _net(0).forward()
    T, B, C = net.V_out.shape
    u = torch.rand((T, B), device="cuda")
    cls, logp, kept = net.draw(u)
    assert cls.shape == (T, B) and logp.shape == (T, B) and bool((kept == C).all())
    last, _, _ = net.draw(u[-1], step=-1)
    assert torch.equal(last, cls[-1])
    cold, _, _ = net.draw(u[-1], torch.zeros(B, device="cuda"), step=T - 1)
    assert cold.cpu().tolist() == [int(rows.order(r)[0]) for r in net.V_out[-1].cpu().numpy()]
    assert snn.SNN_OK == 0


def test_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        import distill
    finally:
        sys.path.pop(0)
    said = []
    first, last, right = distill.run(steps=45, teacher_steps=45, batch=32, hidden=32, say=said.append)
    print("\n".join(said), flush=True)
    assert last < first and len(said) == 4
    assert all(0.0 <= v <= 1.0 for pair in right.values() for v in pair)
