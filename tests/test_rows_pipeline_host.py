"""What the networks keep and hand on around the readout's row operators, on the CPU: the entry points are replaced, and
shapes and arguments are looked at."""
import pytest
import torch

from paper_2105_08810_amd import pipeline, snn


def _network(kind, T, B, C, mode=0):
    labels = torch.zeros(B, dtype=torch.int32)
    if kind == "dense":
        return pipeline.Network(X=torch.zeros((T, B, 6), dtype=torch.uint8), Ws=[torch.zeros((6, 4))],
                                W_out=torch.zeros((4, C)), alphas=[0.9], alpha_out=0.9, labels=labels, loss_mode=mode)
    return pipeline.ConvNetwork(X=torch.zeros((T, B, 4, 4, 1), dtype=torch.uint8), Wc=torch.zeros((3, 3, 1, 2)),
                                W_out=torch.zeros((8, C)), alpha=0.9, alpha_out=0.9, labels=labels, loss_mode=mode)


@pytest.fixture
def calls(monkeypatch):
    """The weights that readout_distill is called with."""
    seen = []

    def readout_ce(V, labels, mode, dense=False):
        n = V.shape[1] * V.shape[2] if mode == 0 else V.numel()
        eps_dense = torch.zeros(V.shape) if dense else None
        return snn.Csr(torch.zeros(V.shape[0] * V.shape[1] + 1, dtype=torch.int32), None, None, None, n), torch.zeros(n), \
            torch.zeros(1), eps_dense

    def readout_distill(z, ids, vals, lse=None, tau=1.0, weight=None, grad=None, accumulate=False):
        assert grad.shape == z.shape and accumulate
        seen.append(weight)
        return torch.zeros(1), torch.zeros(z.shape[:-1]), grad

    monkeypatch.setattr(snn, "readout_ce", readout_ce)
    monkeypatch.setattr(snn, "readout_distill", readout_distill)
    return seen


def _record(T, B):
    return pipeline.Record(torch.zeros((T, B, 1), dtype=torch.int32), torch.zeros((T, B, 1)), None, 1.0)


def _is_every_entry(csr, T, B, C):
    assert csr.row_ptr.tolist() == list(range(0, T * B * C + 1, C))
    assert csr.col_idx.tolist() == list(range(C)) * (T * B)
    assert csr.capacity == T * B * C and csr.nnz() == T * B * C


@pytest.mark.parametrize("kind", ["dense", "conv"])
def test_entries_follow_the_shape(calls, kind):
    """One network object through batches of other sizes: the CSR of every entry is that of the present V_out."""
    net = _network(kind, 3, 2, 5)
    for T, B, C in ((3, 2, 5), (4, 7, 5), (2, 1, 5), (3, 2, 5), (5, 3, 2)):  # the last: as many entries, other rows
        other = _network(kind, T, B, C)
        net.X, net.W_out, net.labels = other.X, other.W_out, other.labels
        net.allocate()
        csr, eps, _, _, _ = net.readout_distilled(pipeline.Distill(_record(T, B)))
        _is_every_entry(csr, T, B, C)
        assert eps.numel() == T * B * C
        assert net.readout_distilled(pipeline.Distill(_record(T, B)))[0] is csr  # kept from step to step


def test_entries_follow_a_replaced_readout(calls):
    net = _network("dense", 3, 2, 5)
    for T, B, C in ((3, 2, 5), (6, 2, 5), (3, 5, 2)):
        net.V_out = torch.zeros((T, B, C))
        _is_every_entry(net.readout_distilled(pipeline.Distill(_record(T, B)))[0], T, B, C)


@pytest.mark.parametrize("kind", ["dense", "conv"])
def test_allocate_drops_the_entries(calls, kind):
    net = _network(kind, 3, 2, 5).allocate()
    net.readout_distilled(pipeline.Distill(_record(3, 2)))
    assert net._every is not None
    assert net.allocate()._every is None


def test_allocate_drops_the_active_sets(monkeypatch):
    """The bitsets of the active sets are as long as the batch: a forward after allocate() for a longer one makes new
    ones. (Forwards replaced: they are given the bitsets they would write.)"""
    given = []
    monkeypatch.setattr(snn, "snn_lif_forward_traces", lambda *a: given.append(a[14].numel()))
    monkeypatch.setattr(snn, "snn_lif_forward", lambda *a: None)
    net = _network("dense", 3, 2, 5)
    for T, B in ((3, 2), (40, 70), (2, 1)):
        net.X = torch.zeros((T, B, 6), dtype=torch.uint8)
        net.allocate().forward(0.5)
        assert given[-1] == snn.snn_active_bits_words(T, B, 4)
        assert net.bits_bth == 0.5


@pytest.mark.parametrize("kind", ["dense", "conv"])
def test_scale_is_a_factor_of_any_weight(calls, kind):
    net = _network(kind, 3, 2, 5).allocate()
    rec, weight = _record(3, 2), torch.rand((3, 2))
    for w, scale in ((None, 1.0), (None, 0.5), (weight, 1.0), (weight, 0.5), (weight, 0.0)):
        net.readout_distilled(pipeline.Distill(rec, w, scale))
        got = torch.full((3, 2), 1 / 6) if calls[-1] is None else calls[-1]
        want = (torch.full((3, 2), 1 / 6) if w is None else w) * scale
        assert got.shape == (3, 2) and torch.allclose(got, want, rtol=1e-6, atol=0.0)
    assert torch.equal(rec.vals, _record(3, 2).vals) and bool((weight > 0).any())  # neither is changed
