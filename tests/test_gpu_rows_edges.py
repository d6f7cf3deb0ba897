"""The operators on rows of logits and the networks around them at their edges: what is kept between calls, logits at a
type's lowest value, rows that are not finite, more rows than one launch counts, the longest rows."""
import math

import numpy as np
import pytest
import torch

from oracle import rows
from paper_2105_08810_amd import pipeline, snn
from synth import CONFIGS, make_inputs

pytestmark = pytest.mark.gpu

INF = math.inf
U = 2.0 ** -24


# ---------------------------------------------------------------- what a network keeps

def _teacher_record(net):
    g = torch.Generator(device="cuda").manual_seed(5)
    T, B, C = net.V_out.shape
    vals, ids = torch.randn((T, B, C), generator=g, device="cuda").topk(2, dim=2)
    return pipeline.Record(ids.to(torch.int32).contiguous(), vals.contiguous(), None, 1.0)


def _is_every_entry(csr, T, B, C):
    assert csr.row_ptr.cpu().tolist() == list(range(0, T * B * C + 1, C))
    assert csr.col_idx.cpu().tolist() == list(range(C)) * (T * B)
    assert csr.capacity == T * B * C and csr.nnz() == T * B * C


def test_entries_made_in_a_capture_are_the_graphs():
    """A CSR first made while a stream is captured is filled by replays alone: an eager call before the first replay
    makes its own, and both stay right from then on."""
    net = pipeline.from_inputs(make_inputs(CONFIGS["tiny"]))
    net.loss_mode = 0
    net.forward()
    T, B, C = net.V_out.shape
    d = pipeline.Distill(_teacher_record(net))
    g = pipeline.Graphed(lambda: net.readout_distilled(d))
    assert net._every is None
    want = net.readout_distilled(d)
    _is_every_entry(want[0], T, B, C)
    for _ in range(3):
        csr, eps, ce, _, kd = g()
        torch.cuda.synchronize()
        _is_every_entry(csr, T, B, C)
        again = net.readout_distilled(d)
        _is_every_entry(again[0], T, B, C)
        assert torch.equal(eps, again[1]) and torch.equal(ce, again[2]) and torch.equal(kd, again[4])
        assert torch.equal(eps, want[1])


def test_conv_steps_of_two_batch_sizes():
    """One network object through a batch, a larger one and a smaller one gives each the gradients that a fresh network
    gives it."""
    inp = make_inputs(CONFIGS["conv"], list(range(4)))
    X = torch.from_numpy(inp.X).cuda()
    labels = torch.from_numpy(inp.labels.astype("int32")).cuda()
    T = 10

    def fresh():
        g = torch.Generator(device="cuda").manual_seed(0)
        return pipeline.ConvNetwork(X=None, Wc=torch.randn((3, 3, 1, 8), generator=g, device="cuda"),
                                    W_out=torch.randn((14 * 14 * 8, 10), generator=g, device="cuda") * 0.05, alpha=0.9,
                                    alpha_out=0.9, labels=None, loss_mode=0)

    def step(net, B):
        net.X, net.labels = X[:T, :B].reshape(T, B, 28, 28, 1).contiguous(), labels[:B].contiguous()
        net.allocate()
        record = _teacher_record(net)  # by the shape alone
        return net.train_step(pipeline.Adam(net.params(), lr=0.0), 0.5, distill=pipeline.Distill(record))

    one = fresh()
    for B in (2, 4, 1):
        got, want = step(one, B), step(fresh(), B)
        assert float(got["kd"]) == float(want["kd"]) > 0
        for a, b in zip(got["grads"], want["grads"]):
            assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max())
