"""The operators on token sequences at sizes whose offsets pass 32 bits and whose rows take several launches, against 64 bits on
the device: rows at the ends and beside the lines between launches, sums over all rows in runs."""
import math

import pytest
import torch

from paper_2105_08810_amd import snn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16 = 2.0 ** -8  # half a step
INT = torch.int32


@pytest.fixture(autouse=True)
def free_after():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_large_embedding():
    """A table of more than 2^31 values, its last rows among those picked."""
    V, N = (1 << 18) + 3, 8200
    E = torch.empty((V, N), dtype=torch.bfloat16, device="cuda").normal_(generator=gen(1))
    ids = torch.tensor([V - 1, 0, V, (1 << 31) // N, -1, (1 << 31) // N + 1, V - 1, 5], dtype=INT, device="cuda")
    live = (ids >= 0) & (ids < V)
    out = snn.embed(E, ids, 2.0)
    assert torch.equal(out, torch.where(live[:, None], E[ids.clamp(0, V - 1).long()] * 2, 0.0))
    E.fill_(1.0)
    dE = snn.embed_grad(ids, out, V, 0.5, dE=E)
    assert int(dE.any(1).sum()) == 5
    for v in ids[live].unique().tolist():
        want = out[ids == v].double().sum(0) * 0.5
        assert bool(((dE[v].double() - want).abs() <= (BF16 + 4 * U) * want.abs() + 1e-38).all())


def test_many_rows_of_an_embedding():
    """More rows than a launch, and more than 2^31 values of them."""
    R, V, N = (1 << 22) + 7, 700, 520
    E = torch.randn((V, N), generator=gen(2), device="cuda").to(torch.bfloat16)
    ids = torch.randint(-1, V + 1, (R,), generator=gen(3), device="cuda").to(INT)
    live = (ids >= 0) & (ids < V)
    out = snn.embed(E, ids)
    for r0 in (0, (1 << 22) - 9, R - 16):
        at = ids[r0:r0 + 16].clamp(0, V - 1).long()
        assert torch.equal(out[r0:r0 + 16], torch.where(live[r0:r0 + 16, None], E[at], 0.0))
    dE = snn.embed_grad(ids, out, V)
    # every row of a token is the same, so its sum is their number times it: in float32 over 128 of them
    n = torch.bincount(ids[live].long(), minlength=V).double()[:, None]
    want = n * E.double()
    assert bool(((dE.double() - want).abs() <= (BF16 + 131 * U) * want.abs()).all())


def test_many_rows_of_a_norm():
    R, N = (1 << 21) + 9, 1030
    x = torch.empty((R, N), dtype=torch.bfloat16, device="cuda").normal_(0.5, 2.0, generator=gen(4))
    gamma = 1 + 0.1 * torch.randn(N, generator=gen(5), device="cuda")
    y, mean, rstd = snn.layer_norm(x, gamma)
    dx, dgamma, dbeta = snn.layer_norm_grad(y, x, gamma, mean, rstd)  # dy = y
    g64 = gamma.double()
    sums = torch.zeros((4, N), dtype=torch.float64, device="cuda")
    for r0 in range(0, R, 1 << 18):
        s = slice(r0, min(R, r0 + (1 << 18)))
        h = (x[s].double() - mean[s].double()[:, None]) * rstd[s].double()[:, None]
        dy = y[s].double()
        sums += torch.stack([(dy * h).sum(0), dy.sum(0), (dy * h).abs().sum(0), dy.abs().sum(0)])
        if r0 == 0 or r0 >= (1 << 21) - (1 << 18):
            want = h * g64
            assert bool(((dy - want).abs() <= (BF16 + 100 * U) * want.abs() + 100 * U).all())
            a = dy * g64
            want = rstd[s].double()[:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
            top = rstd[s].double()[:, None] * (a.abs() + a.abs().mean(1, keepdim=True) + h.abs() * (a * h).abs().mean(1, keepdim=True))
            assert bool(((dx[s].double() - want).abs() <= BF16 * want.abs() + 100 * U * top).all())
    # a group's rows in one chain of float32, at most R / 512 of them, x - mean rounded once
    chain = R // 512 + 60
    assert bool(((dgamma.double() - sums[0]).abs() <= chain * U * sums[2]).all())
    assert bool(((dbeta.double() - sums[1]).abs() <= chain * U * sums[3]).all())


@pytest.mark.parametrize("dtype,C", [("f32", 2), ("bf16", 2), ("f16", 2), ("f32", 150), ("bf16", 150)])
def test_most_rows_of_cross_entropy(dtype, C):
    """2^24 rows, the most that there may be; with 150 classes their logits are more than 2^31 values."""
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    R, H = 1 << 24, 3
    x = torch.randn((R, H), generator=gen(6), device="cuda").to(dt)
    W = torch.randn((H, C), generator=gen(7), device="cuda").to(dt)
    t = torch.randint(-1, C, (R,), generator=gen(8), device="cuda").to(INT)
    w = torch.ones(R, device="cuda")
    loss, row_loss, dx, dW = snn.linear_ce(x, W, t, w)
    u = {"f32": U, "bf16": BF16, "f16": 2.0 ** -11}[dtype]
    one = 0.0 if dtype == "f32" else u
    W64 = W.double()
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    ref, size = torch.zeros_like(W64), torch.zeros_like(W64)
    for r0 in range(0, R, 1 << 21):
        s = slice(r0, r0 + (1 << 21))
        live, X = t[s] >= 0, x[s].double()
        at = t[s].clamp_min(0).long()[:, None]
        z = X @ W64
        others = z.scatter(1, at, -math.inf)
        rest = torch.logsumexp(others, 1, keepdim=True)
        zt = z.gather(1, at)
        lse = torch.logaddexp(rest, zt)
        row = torch.where(live, torch.nn.functional.softplus(rest - zt)[:, 0], 0.0)
        ez = 2 * (H + 4) * U * (X.abs() @ W64.abs()).amax(1) + (C / 64 + 100) * U
        assert bool(((row_loss[s].double() - row).abs() <= 2 * ez + 8 * U * (1 + row)).all())
        total += row.sum()
        dz = torch.exp(others - lse).scatter_(1, at, -torch.exp(rest - lse)) * live[:, None]
        e = dz.abs() * (2 * ez[:, None] + one) + live[:, None] * (0.0 if dtype == "f32" else 2.0 ** -40)
        want = dz @ W64.T
        tol = e @ W64.abs().T + 2 * (C + 4) * U * (dz.abs() @ W64.abs().T)
        assert bool(((dx[s].double() - want).abs() <= tol + u * (want.abs() + tol) + 2.0 ** -25).all())
        ref += X.T @ dz
        size += X.abs().T @ e + 4096 * U * (X.abs().T @ dz.abs())
    assert abs(float(loss) - float(total)) < 1e-5 * float(total)
    if dtype == "f16" and float(ref.abs().max()) > 65504:
        return  # beyond its range
    # sums of 2^24 terms: K slices of the product, a few thousand roundings deep where they are not of both signs
    assert bool(((dW.double() - ref).abs() <= size + u * (ref.abs() + size)).all())
