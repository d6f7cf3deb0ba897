"""Networks on tokens: what is refused before any device call."""
import pytest
import torch

from paper_2105_08810_amd import pipeline


def network(tokens=True, every=True, norm=False):
    X = torch.zeros((4, 3), dtype=torch.int32) if tokens else torch.zeros((4, 3, 7), dtype=torch.uint8)
    labels = torch.zeros((4, 3) if every else (3,), dtype=torch.int32)
    n = pipeline.Norm(torch.ones(5), torch.zeros(5)) if norm else None
    return pipeline.Network(X=X, Ws=[torch.zeros((7, 5))], W_out=torch.zeros((5, 2)), alphas=[0.9], alpha_out=0.9,
                            labels=labels, loss_mode=1, norm_in=n)


def test_kinds():
    assert network().tokens and network().every_step
    assert not network(tokens=False).tokens and not network(every=False).every_step
    assert len(network(norm=True).params()) == 4 and len(network().params()) == 2


def test_norm_needs_tokens():
    with pytest.raises(ValueError, match="norm_in"):
        network(tokens=False, norm=True)


@pytest.mark.parametrize("kw", [dict(), dict(every=False), dict(tokens=False)])
def test_no_dense_backward(kw):
    net = network(**kw)
    with pytest.raises(ValueError, match="dense"):
        net.dense_backward(0.2)
    with pytest.raises(ValueError, match="dense"):
        net.train_step(None, 0.2, sparse=False)


def test_one_label_paths():
    net = network()
    with pytest.raises(ValueError, match="every step"):
        net.readout()
    with pytest.raises(ValueError, match="every step"):
        net.train_step(None, 0.2, distill=pipeline.Distill(None))
    with pytest.raises(ValueError, match="forward"):
        net.membrane()
