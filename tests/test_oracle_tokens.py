"""The oracle of the operators on sequences of tokens, against autograd in 64 bits and differences."""
import numpy as np
import pytest
import torch

from oracle import tokens


def _leaf(a):
    return torch.tensor(a, dtype=torch.float64, requires_grad=True)


def test_embedding():
    rng = np.random.default_rng(1)
    E, ids = rng.standard_normal((7, 5)), np.array([3, -1, 0, 3, 7, 6, 3])
    g = rng.standard_normal((7, 5))
    t = _leaf(E)
    ok = torch.tensor((ids >= 0) & (ids < 7))
    out = t[torch.tensor(np.where(ok, ids, 0))] * ok[:, None] * 2.5
    assert np.allclose(tokens.embed(E, ids, 2.5), out.detach().numpy(), rtol=1e-15, atol=0)
    (out * torch.tensor(g)).sum().backward()
    dE, bound, n = tokens.embed_grad(ids, g, 7, 2.5)
    assert np.allclose(dE, t.grad.numpy(), rtol=1e-13, atol=1e-13)
    assert n.tolist() == [1, 0, 0, 3, 0, 0, 1] and (np.abs(dE) <= bound + 1e-12).all()


@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm(affine):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((6, 9)) * 3 + 1, rng.standard_normal((6, 9))
    gamma, beta = (rng.standard_normal(9), rng.standard_normal(9)) if affine else (None, None)
    tx = _leaf(x)
    tg, tb = (_leaf(gamma), _leaf(beta)) if affine else (None, None)
    ty = torch.nn.functional.layer_norm(tx, (9,), tg, tb, eps=1e-3)
    y, mean, rstd = tokens.layer_norm(x, gamma, beta, 1e-3)
    assert np.allclose(y, ty.detach().numpy(), rtol=1e-12, atol=1e-12)
    (ty * torch.tensor(dy)).sum().backward()
    (dx, dgamma, dbeta), _ = tokens.layer_norm_grad(dy, x, gamma, mean, rstd)
    assert np.allclose(dx, tx.grad.numpy(), rtol=1e-11, atol=1e-12)
    if affine:
        assert np.allclose(dgamma, tg.grad.numpy(), rtol=1e-11, atol=1e-12)
        assert np.allclose(dbeta, tb.grad.numpy(), rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("weighted", [False, True])
def test_linear_ce(weighted):
    rng = np.random.default_rng(3)
    x, W = rng.standard_normal((8, 6)), rng.standard_normal((6, 11))
    t = np.array([0, 10, -1, 4, 11, 4, 4, 2])
    w = np.array([0.5, 0.0, 1.0, 0.25, 1.0, 2.0, 0.1, 0.3]) if weighted else None
    r = tokens.linear_ce(x, W, t, w)
    tx, tw = _leaf(x), _leaf(W)
    rows = torch.nn.functional.cross_entropy(tx @ tw, torch.tensor(np.where((t >= 0) & (t < 11), t, -100)),
                                             ignore_index=-100, reduction="none")
    live = (t >= 0) & (t < 11)
    loss = (rows * torch.tensor(w if weighted else live / live.sum())).sum()
    assert r["loss"] == pytest.approx(float(loss), rel=1e-13)
    loss.backward()
    assert np.allclose(r["dx"], tx.grad.numpy(), rtol=1e-12, atol=1e-14)
    assert np.allclose(r["dW"], tw.grad.numpy(), rtol=1e-12, atol=1e-14)
    d = rng.standard_normal(W.shape)  # and against differences
    h = 1e-6
    diff = (tokens.linear_ce(x, W + h * d, t, w)["loss"] - tokens.linear_ce(x, W - h * d, t, w)["loss"]) / (2 * h)
    assert diff == pytest.approx((r["dW"] * d).sum(), rel=1e-7)


def test_leak_grad():
    rng = np.random.default_rng(4)
    i, g, alpha = rng.standard_normal((9, 2, 3)), rng.standard_normal((9, 2, 3)), 0.7
    ti = _leaf(i)
    u = [torch.zeros(2, 3, dtype=torch.float64)]
    for t in range(8):
        u.append(alpha * u[-1] + ti[t])
    (torch.stack(u) * torch.tensor(g)).sum().backward()
    assert np.allclose(tokens.leak_grad(g, alpha), ti.grad.numpy(), rtol=1e-13, atol=1e-14)
