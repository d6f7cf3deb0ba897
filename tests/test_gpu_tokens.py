"""The operators of a network on sequences of tokens against the float64 oracle: every type, sizes from one on, padded and
misaligned rows, rows without a token or a target, runs of one token over many blocks, long rows, several pieces."""
import functools
import math

import numpy as np
import pytest
import torch

from oracle import tokens
from paper_2105_08810_amd import pipeline, snn

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# relative rounding of a result to its type (half a step), and that of its smallest numbers
ROUND = {"f32": (2.0 ** -24, 2.0 ** -149), "bf16": (2.0 ** -8, 2.0 ** -133), "f16": (2.0 ** -11, 2.0 ** -25)}
U = 2.0 ** -24
INF, NAN = math.inf, math.nan


def rows_on(z, dtype, ld=None, lead=0):
    """z [R, C] as rows of dtype in rows of ld elements, `lead` elements past an aligned address, NaN around them."""
    R, C = z.shape
    ld = C if ld is None else ld
    full = torch.full((R * ld + lead,), NAN, dtype=DTYPES[dtype], device="cuda")
    view = full[lead:].view(R, ld)[:, :C]
    view.copy_(torch.from_numpy(np.ascontiguousarray(z)).cuda())
    return view


def host(t):
    return t.detach().double().cpu().numpy()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def close(got, want, tol, what):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / tol)} of the tolerance"


# ---------------------------------------------------------------- embedding

LAYOUTS = [(0, 0), (3, 1), (8, 0)]  # elements added to a row, elements past an aligned address


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V,N", [(1, 1, 1), (5, 3, 7), (64, 50, 64), (33, 1000, 300), (7, 20, 1027), (300, 11, 16)])
@pytest.mark.parametrize("pad,lead", LAYOUTS)
def test_embed(dtype, R, V, N, pad, lead):
    rng = np.random.default_rng(R + V + N)
    E = rows_on(rng.standard_normal((V, N)), dtype, N + pad, lead)
    ids = rng.integers(-1, V + 1, R)
    out = rows_on(np.zeros((R, N)), dtype, N + pad, lead)
    snn.embed(E, ids := ints(ids), 1.7, out=out)
    E32 = E.float()
    ok = ((ids >= 0) & (ids < V))[:, None]
    want = torch.where(ok, E32[ids.clamp(0, V - 1).long()] * torch.tensor(1.7, device="cuda"), 0.0).to(DTYPES[dtype])
    assert torch.equal(out, want)  # one product in float32, rounded once
    assert torch.equal(snn.embed(E, ids.view(1, R), 1.7), want.view(1, R, N))
    around = torch.as_strided(out, (R, N + pad), (N + pad, 1))[:R - 1, N:] if R > 1 else out[:, N:]
    assert around.isnan().all()


def _ids(rng, R, V, kind):
    if kind == "one":
        return np.full(R, V // 2)
    if kind == "none":
        return np.where(rng.random(R) < 0.5, -1, V)
    if kind == "zipf":
        return np.minimum(np.exp(rng.random(R) * np.log(V)).astype(int), V) - 1
    if kind == "sorted":
        return np.sort(rng.integers(0, V, R))
    ids = rng.integers(0, V, R)
    ids[rng.random(R) < 0.1] = -1
    return ids


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,V,N,kind", [(1, 1, 1, "one"), (1, 300, 9, "any"), (40, 7, 33, "any"), (64, 64, 8, "none"),
                                        (500, 90, 264, "zipf"), (1000, 3, 16, "sorted"), (777, 5, 1030, "one"),
                                        (8192, 600, 12, "zipf"), (8193, 600, 12, "zipf"), (20000, 1, 5, "one"),
                                        (12345, 513, 24, "any"), (9000, 300000, 3, "zipf"), (40000, 70, 40, "sorted"),
                                        (16384, 2000, 8, "zipf"), (16385, 2000, 8, "zipf")])
def test_embed_grad(dtype, accumulate, R, V, N, kind):
    rng = np.random.default_rng(R + N)
    ids = _ids(rng, R, V, kind)
    dout = rows_on(rng.standard_normal((R, N)), dtype, N + 3, 1)
    if kind != "one" and kind != "sorted":
        dout[torch.from_numpy((ids < 0) | (ids >= V)).cuda()] = NAN  # rows without a token are not used
    before = rng.standard_normal((V, N))
    dE = rows_on(before, dtype, N + 5, 2)
    start = host(dE)
    snn.embed_grad(ints(ids), dout, V, 0.75, dE=dE, accumulate=accumulate)
    want, bound, n = tokens.embed_grad(ids, np.nan_to_num(host(dout)), V, 0.75)
    u, least = ROUND[dtype]
    if accumulate:
        want, bound = want + start, bound + np.abs(start)
        same = n == 0
        assert np.array_equal(host(dE)[same], start[same])
    # n additions in float32 in some order, the product (and the sum with what was there), one rounding
    close(dE, want, (n[:, None] + 3) * U * bound + u * np.abs(want) + least, "dE")
    again = rows_on(before, dtype, N + 5, 2)
    snn.embed_grad(ints(ids), dout, V, 0.75, dE=again, accumulate=accumulate)
    assert torch.equal(again, dE)


# ---------------------------------------------------------------- layer norm

@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"),
                                             ("bf16", "f32"), ("f16", "bf16"), ("f32", "f16"), ("f16", "f32"),
                                             ("bf16", "f16")])
@pytest.mark.parametrize("R,N", [(1, 1), (3, 2), (37, 64), (5, 100), (70, 257), (3, 1024), (9, 2050), (2, 4099), (3, 8192),
                                 (2, 16400), (2, 33001)])
@pytest.mark.parametrize("affine,pad,lead", [("both", 0, 0), ("gamma", 3, 1), ("none", 8, 0), ("beta", 0, 3)])
def test_layer_norm(x_dtype, y_dtype, R, N, affine, pad, lead):
    rng = np.random.default_rng(R + N)
    x = rows_on(rng.standard_normal((R, N)) * 2 + 0.7, x_dtype, N + pad, lead)
    gamma = 1 + 0.3 * rng.standard_normal(N).astype(np.float32) if affine in ("both", "gamma") else None
    beta = rng.standard_normal(N).astype(np.float32) if affine in ("both", "beta") else None
    on = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    y = rows_on(np.zeros((R, N)), y_dtype, N + pad, lead)
    _, mean, rstd = snn.layer_norm(x, on(gamma), on(beta), 1e-3, out=y)
    hx = host(x)
    want, m, k = tokens.layer_norm(hx, gamma, beta, 1e-3)
    # a float32 sum of N terms is n roundings deep: the vectors of a lane, then a tree over the lanes
    n = (N + 1023) // 1024 * 4 + 32
    ax = np.abs(hx).mean(1)
    close(mean, m, (n + 1) * U * ax + 1e-30, "mean")
    off = (n + 2) * U * (ax + np.abs(hx).max(1))  # of x - mean
    # sum of squares: n + 2 roundings and what the mean brings (its square is far below); the root halves it
    krel = (n + 6) * U + (k * off) ** 2
    close(rstd, k, krel * k, "rstd")
    g = np.ones(N) if gamma is None else np.abs(gamma)
    b = np.zeros(N) if beta is None else np.abs(beta)
    h = np.abs(hx - m[:, None]) * k[:, None]
    tol = g * (off * k)[:, None] + g * h * (krel[:, None] + 4 * U) + 2 * U * (g * h + b)
    u, least = ROUND[y_dtype]
    close(y, want, tol + u * (np.abs(want) + tol) + least, "y")

    dy = rows_on(rng.standard_normal((R, N)), y_dtype, N + pad, lead)
    dx, dgamma, dbeta = snn.layer_norm_grad(dy, x, on(gamma), mean, rstd)
    (wx, wg, wb), (tx, tg, tb) = tokens.layer_norm_grad(host(dy), hx, gamma, host(mean), host(rstd))
    u, least = ROUND[x_dtype]
    # (x - mean) is rounded once against |x| + |mean|, which h carries into every term
    lost = U * (np.abs(hx) + np.abs(host(mean))[:, None]) * host(rstd)[:, None]
    a = np.abs(host(dy)) * g
    hs = np.abs(hx - host(mean)[:, None]) * host(rstd)[:, None]
    more = host(rstd)[:, None] * (lost * (a * hs).mean(1, keepdims=True) + hs * (a * lost).mean(1, keepdims=True))
    tol = (n + 8) * U * tx + more
    close(dx, wx, tol + u * (np.abs(wx) + tol) + least, "dx")
    chain = R + 40  # at most every row in one chain, the block's groups, then float64
    close(dgamma, wg, chain * U * tg + (np.abs(host(dy)) * lost).sum(0) + 1e-30, "dgamma")
    close(dbeta, wb, chain * U * tb + 1e-30, "dbeta")
    only, none, _ = snn.layer_norm_grad(dy, x, on(gamma), mean, rstd, want_dgamma=False, want_dbeta=False)
    assert torch.equal(only, dx) and none is None
    none, g2, b2 = snn.layer_norm_grad(dy, x, on(gamma), mean, rstd, want_dx=False)
    assert none is None and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)


# a row that ends inside a lane's vector, with an infinity among its last elements: only its own row's sums hold it, once
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N", [3, 9, 68, 257, 1027, 2051, 4099, 8195])
def test_layer_norm_infinite(dtype, N):
    gen = torch.Generator().manual_seed(N)
    x, dy = (torch.randn(3, N, generator=gen).to(DTYPES[dtype]).cuda() for _ in range(2))
    y0, mean0, rstd0 = snn.layer_norm(x)
    dx0, *_ = snn.layer_norm_grad(dy, x, None, mean0, rstd0, want_dgamma=False, want_dbeta=False)
    xi, di = x.clone(), dy.clone()
    xi[1, N - 2] = INF
    di[1, N - 2] = -INF
    y, mean, rstd = snn.layer_norm(xi)
    assert float(mean[1]) == INF and rstd[1].isnan() and y[1, N - 1].isnan()
    assert torch.equal(y[::2], y0[::2]) and torch.equal(mean[::2], mean0[::2]) and torch.equal(rstd[::2], rstd0[::2])
    dx, dgamma, dbeta = snn.layer_norm_grad(di, x, None, mean0, rstd0)
    assert torch.equal(dx[::2], dx0[::2]) and not dx[1].isfinite().any()
    assert host(~dgamma.isfinite()).nonzero()[0].tolist() == [N - 2] and float(dbeta[N - 2]) == -INF


@pytest.mark.parametrize("R,N", [(5000, 40), (3000, 1024), (1500, 2050)])
def test_layer_norm_many_rows(R, N):
    """More rows than groups of lanes: dgamma and dbeta gather over several rows each."""
    rng = np.random.default_rng(N)
    x, dy = (rows_on(rng.standard_normal((R, N)), "f32") for _ in range(2))
    gamma = torch.from_numpy(1 + 0.1 * rng.standard_normal(N).astype(np.float32)).cuda()
    _, mean, rstd = snn.layer_norm(x, gamma)
    dx, dgamma, dbeta = snn.layer_norm_grad(dy, x, gamma, mean, rstd)
    (wx, wg, wb), (tx, tg, tb) = tokens.layer_norm_grad(host(dy), host(x), host(gamma), host(mean), host(rstd))
    chain = -(-R // 1024) + 48  # rows of one of the 1024 blocks and its groups, a few roundings a term
    lost = U * (np.abs(host(x)) + np.abs(host(mean))[:, None]) * host(rstd)[:, None]
    close(dgamma, wg, chain * U * tg + (np.abs(host(dy)) * lost).sum(0), "dgamma")
    close(dbeta, wb, chain * U * tb, "dbeta")
    x64 = torch.from_numpy(host(x)).requires_grad_(True)  # the whole of it, against autograd in 64 bits
    g64 = torch.from_numpy(host(gamma)).requires_grad_(True)
    y64 = torch.nn.functional.layer_norm(x64, (N,), g64, None, 1e-5)
    y64.backward(torch.from_numpy(host(dy)))
    assert np.linalg.norm(host(dx) - x64.grad.numpy()) < 1e-6 * np.linalg.norm(x64.grad.numpy())
    assert np.linalg.norm(host(dgamma) - g64.grad.numpy()) < 1e-5 * np.linalg.norm(g64.grad.numpy())
    again = snn.layer_norm_grad(dy, x, gamma, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dgamma, dbeta)))


# ---------------------------------------------------------------- cross entropy of linear logits

def ce_case(R, H, C, dtype, seed, pad=0, lead=0, dead=0.2, spread=2.0):
    rng = np.random.default_rng(seed)
    x = rows_on(rng.standard_normal((R, H)), dtype, H + pad, lead)
    W = rows_on(rng.standard_normal((H, C)) * spread / math.sqrt(H), dtype, C + pad, lead)
    t = rng.integers(0, C, R)
    t[rng.random(R) < dead] = -1
    return rng, x, W, t


def check_ce(x, W, t, weight, out, dtype):
    loss, row_loss, dx, dW = out
    r = tokens.linear_ce(np.nan_to_num(host(x)), host(W), t, weight)
    R, H = x.shape
    C = W.shape[1]
    u, least = ROUND[dtype]
    # z: H products summed in float32, the matrix cores' steps rounded towards zero (a whole step, 2 U)
    dz = 2 * (H + 4) * U * r["z_bound"]
    # lse: the sum of exponentials (C roundings at most, each exponential two and its argument's), a logarithm; all three
    # terms of the loss rounded against the largest logit's size
    top = r["z_bound"]
    tol = 2 * dz + (C / 64 + 40) * U + 6 * U * (top + np.abs(r["row_loss"]) + 1)
    live = r["live"]
    assert not host(row_loss)[~live].any()
    close(host(row_loss), r["row_loss"], tol, "row_loss")
    close(host(loss), r["loss"], (np.abs(r["w"]) * tol).sum() + 2 * U * (np.abs(r["w"]) * r["row_loss"]).sum() + 1e-37,
          "loss")
    if dx is None:
        return r
    # dz: its exponent's error, a few roundings; in 16 bits one rounding to the type
    one = u if dtype != "f32" else 0.0
    w = np.abs(r["w"])[:, None]
    e = w * r["p"] * (2 * dz[:, None] + (C / 64 + 40) * U + 12 * U * (top[:, None] + 1)) + (4 * U + one) * np.abs(r["dz"])
    # in 16 bits dz / ref (ref the largest weight) is formed by the hardware's exponential, whose results below float32's
    # smallest normal number 2^-126 are 0, and kept in a type with half a step of at most 2^-126 (bfloat16: 2^-134; float16,
    # raised by 2^15: 2^-25 / 2^15 = 2^-40)
    if dtype != "f32":
        e = e + live[:, None] * w.max() * (2.0 ** -126 if dtype == "bf16" else 2.0 ** -40)
    absW, X = np.abs(host(W)), np.abs(r["X"])
    tol = e @ absW.T + 2 * (C + 4) * U * (np.abs(r["dz"]) @ absW.T)
    close(dx, r["dx"], tol + u * (np.abs(r["dx"]) + tol) + least, "dx")
    assert not host(dx)[~live].any()
    tol = X.T @ e + 2 * (R + 4) * U * (X.T @ np.abs(r["dz"]))
    close(dW, r["dW"], tol + u * (np.abs(r["dW"]) + tol) + least, "dW")
    return r


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,H,C", [(1, 1, 1), (1, 8, 2), (3, 5, 7), (64, 64, 64), (130, 200, 10), (257, 33, 300), (20, 130, 1000),
                                   (300, 260, 513), (1, 256, 4097), (1000, 17, 3)])
@pytest.mark.parametrize("pad,lead", [(0, 0), (3, 1), (8, 8)])
def test_linear_ce(dtype, R, H, C, pad, lead):
    rng, x, W, t = ce_case(R, H, C, dtype, R + H + C, pad, lead, dead=0.2 if R > 1 else 0.0)
    x[torch.from_numpy(t < 0).cuda()] = NAN  # rows without a target are not read
    out = snn.linear_ce(x, W, ints(t))
    check_ce(x, W, t, None, out, dtype)
    w = rng.random(R).astype(np.float32)
    w[rng.random(R) < 0.3] = 0.0
    out = snn.linear_ce(x, W, ints(t), torch.from_numpy(w).cuda())
    check_ce(x, W, t, w, out, dtype)
    loss, row_loss, dx, dW = snn.linear_ce(x, W, ints(t), torch.from_numpy(w).cuda(), want_grad=False)
    assert dx is None and dW is None
    assert torch.equal(row_loss, out[1]) and torch.equal(loss, out[0])


# few classes of more rows: dW in slices of the rows, of a number that divides them and not
@pytest.mark.parametrize("R,H,C", [(4097, 7, 3), (5000, 33, 17), (9001, 20, 40), (4500, 300, 64), (4111, 600, 60)])
def test_linear_ce_slices(R, H, C):
    rng, x, W, t = ce_case(R, H, C, "f32", R, 3, 1)
    x[torch.from_numpy(t < 0).cuda()] = NAN
    out = snn.linear_ce(x, W, ints(t))
    check_ce(x, W, t, None, out, "f32")
    ws, behind = poisoned(snn.snn_linear_ce_workspace(x.dtype, R, H, C, True))
    assert all(torch.equal(p, q) for p, q in zip(snn.linear_ce(x, W, ints(t), ws=ws), out)) and bool((behind == 255).all())
    loss, *_ = snn.linear_ce(x, W, ints(t), want_grad=False)
    assert torch.equal(loss, out[0])


# around every number of classes at which lanes take more of them at once, rows and columns that end inside a run of 16
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [4, 15, 16, 17, 19, 31, 32, 33, 35, 61, 63, 65, 66, 95, 97, 111, 113, 127, 128, 129])
def test_linear_ce_classes(dtype, C):
    rng, x, W, t = ce_case(37, 41, C, dtype, C, 3, 1)
    x[torch.from_numpy(t < 0).cuda()] = NAN
    w = rng.random(37).astype(np.float32)
    check_ce(x, W, t, w, snn.linear_ce(x, W, ints(t), torch.from_numpy(w).cuda()), dtype)


# the widest rows: 128 and more classes, and few
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [5, 130])
def test_linear_ce_widest(dtype, C):
    _, x, W, t = ce_case(3, 1 << 16, C, dtype, C, dead=0.0)
    check_ce(x, W, t, None, snn.linear_ce(x, W, ints(t)), dtype)


# more rows than one block counts, with and without weights
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [6, 150])
@pytest.mark.parametrize("weighted", [False, True])
def test_linear_ce_many_rows(dtype, C, weighted):
    R = 33000
    rng, x, W, t = ce_case(R, 8, C, dtype, C, dead=0.3)
    x[torch.from_numpy(t < 0).cuda()] = NAN
    w = np.where(rng.random(R) < 0.3, 0.0, rng.random(R)).astype(np.float32) if weighted else None
    check_ce(x, W, t, w, snn.linear_ce(x, W, ints(t), None if w is None else torch.from_numpy(w).cuda()), dtype)


def poisoned(nbytes):
    """A workspace of NaN, and what lies behind it."""
    ws = torch.full((nbytes + 4096,), 255, dtype=torch.uint8, device="cuda")
    return ws[:nbytes], ws[nbytes:]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,H,C", [(1, 1, 1), (65, 24, 10), (300, 37, 101), (5000, 37, 101), (77, 70, 300), (500, 130, 1027),
                                   (2900, 9, 47001)])
def test_linear_ce_workspace(dtype, R, H, C):
    """What the workspace held before does not matter, and nothing behind it is written."""
    _, x, W, t = ce_case(R, H, C, dtype, 4, dead=0.2 if R > 1 else 0.0)
    want = snn.linear_ce(x, W, ints(t))
    ws, behind = poisoned(snn.snn_linear_ce_workspace(x.dtype, R, H, C, True))
    got = snn.linear_ce(x, W, ints(t), ws=ws)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and bool((behind == 255).all())
    ws, behind = poisoned(snn.snn_linear_ce_workspace(x.dtype, R, H, C, False))
    got = snn.linear_ce(x, W, ints(t), ws=ws, want_grad=False)
    assert all(torch.equal(p, q) for p, q in zip(got[:2], want)) and bool((behind == 255).all())
    with pytest.raises(snn.SnnError):
        snn.linear_ce(x, W, ints(t), ws=ws[:-1], want_grad=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_workspaces(dtype):
    gen = torch.Generator().manual_seed(1)
    for R, V, N in [(1, 1, 1), (700, 90, 33), (17000, 600, 5)]:
        ids = torch.randint(-1, V, (R,), generator=gen, dtype=torch.int32).cuda()
        dout = torch.randn(R, N, generator=gen).to(DTYPES[dtype]).cuda()
        ws, behind = poisoned(snn.snn_embed_grad_workspace(dout.dtype, V, N, R))
        assert torch.equal(snn.embed_grad(ids, dout, V, ws=ws), snn.embed_grad(ids, dout, V)) and bool((behind == 255).all())
        with pytest.raises(snn.SnnError):
            snn.embed_grad(ids, dout, V, ws=ws[:-1])
    for R, N in [(1, 1), (700, 33), (300, 1030), (100, 4100), (20, 40000)]:
        x, dy = (torch.randn(R, N, generator=gen).to(DTYPES[dtype]).cuda() for _ in range(2))
        _, mean, rstd = snn.layer_norm(x)
        ws, behind = poisoned(snn.snn_layer_norm_grad_workspace(x.dtype, x.dtype, R, N))
        got, want = snn.layer_norm_grad(dy, x, None, mean, rstd, ws=ws), snn.layer_norm_grad(dy, x, None, mean, rstd)
        assert all(torch.equal(p, q) for p, q in zip(got, want)) and bool((behind == 255).all())
        with pytest.raises(snn.SnnError):
            snn.layer_norm_grad(dy, x, None, mean, rstd, ws=ws[:-1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_ce_one_gradient(dtype):
    """Either gradient alone, written into rows of a wider tensor, what is around them untouched."""
    _, x, W, t = ce_case(150, 72, 290, dtype, 5, 3, 1)
    _, _, dx, dW = snn.linear_ce(x, W, ints(t))
    loss, ws = torch.empty(1, device="cuda"), snn.workspace(snn.snn_linear_ce_workspace(x.dtype, 150, 72, 290, True))
    out = rows_on(np.zeros((150, 72)), dtype, 80, 3)
    snn.snn_linear_ce(x, W, ints(t), None, loss, None, out, None, ws)
    assert torch.equal(out, dx) and torch.as_strided(out, (149, 80), (80, 1))[:, 72:].isnan().all()
    out = rows_on(np.zeros((72, 290)), dtype, 301, 1)
    snn.snn_linear_ce(x, W, ints(t), None, loss, None, None, out, ws)
    assert torch.equal(out, dW) and torch.as_strided(out, (71, 301), (301, 1))[:, 290:].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_ce_without_targets(dtype):
    _, x, W, _ = ce_case(70, 40, 90, dtype, 6)
    x.fill_(NAN)
    t = np.full(70, -1)
    t[3], t[9] = 90, -7
    for out in (snn.linear_ce(x, W, ints(t)), snn.linear_ce(x, W, ints(np.zeros(70)), torch.zeros(70, device="cuda"))):
        assert all(not host(o).any() for o in out)


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_ce_extremes(dtype):
    """A NaN stays in its row's loss and gradient; logits far apart; one class."""
    _, x, W, t = ce_case(20, 16, 50, dtype, 7, dead=0.0)
    x[4, 3] = NAN
    loss, row_loss, dx, _ = snn.linear_ce(x, W, ints(t))
    assert math.isnan(float(loss)) and host(row_loss.isnan()).nonzero()[0].tolist() == [4]
    assert host(dx.isnan().any(1)).nonzero()[0].tolist() == [4]
    x[4, 3] = 0.0
    x *= 100.0  # logits of hundreds: exponentials of most are 0
    check_ce(x, W, t, None, snn.linear_ce(x, W, ints(t)), dtype)
    out = snn.linear_ce(x, W[:, :1], ints(np.zeros(20)))
    assert all(not host(o).any() for o in out)


@pytest.mark.parametrize("dtype,R,H,C", [("f32", 3000, 24, 70000), ("bf16", 3000, 24, 200003), ("f16", 2500, 40, 131072)])
def test_linear_ce_pieces(dtype, R, H, C):
    """More logits than a piece holds, against 64 bits on the device."""
    g = torch.Generator(device="cuda").manual_seed(R)
    x = torch.randn((R, H), generator=g, device="cuda").to(DTYPES[dtype])
    W = (torch.randn((H, C), generator=g, device="cuda") * 0.4).to(DTYPES[dtype])
    t = torch.randint(-1, C, (R,), generator=g, device="cuda").to(torch.int32)
    loss, row_loss, dx, dW = snn.linear_ce(x, W, t)
    live = t >= 0
    z = x.double() @ W.double()
    logp = torch.log_softmax(z, 1)
    want = torch.where(live, -logp.gather(1, t.clamp_min(0).long()[:, None])[:, 0], 0.0)
    assert float((row_loss.double() - want).abs().max()) < 40 * U * float(z.abs().max()) + 2 * H * U * 40
    p = torch.exp(logp)
    p.scatter_add_(1, t.clamp_min(0).long()[:, None], -torch.ones_like(p[:, :1]))
    p *= (live.double() / live.sum())[:, None]
    # relative to the whole: roundings of a random sign each
    u = 4 * ROUND[dtype][0] if dtype != "f32" else 2e-6
    for got, ref in ((dx, p @ W.double().T), (dW, x.double().T @ p)):
        least = ROUND[dtype][1] * math.sqrt(ref.numel())
        assert float((got.double() - ref).norm()) < u * float(ref.norm()) + least


# ---------------------------------------------------------------- the adjoint of the leak

def csr_of(on, with_g=None):
    rp = np.concatenate([[0], on.reshape(-1, on.shape[2]).sum(1).cumsum()]).astype(np.int32)
    col = np.nonzero(on.reshape(-1, on.shape[2]))[1].astype(np.int32)
    g = None if with_g is None else torch.from_numpy(with_g[on].astype(np.float32)).cuda()
    return snn.Csr(ints(rp), ints(col), g, None, len(col))


@pytest.mark.parametrize("T,B,N", [(1, 1, 1), (2, 3, 5), (20, 4, 32), (33, 2, 300), (32, 1, 256), (65, 3, 257), (100, 2, 64),
                                   (500, 1, 40), (34, 2, 70), (129, 1, 300), (130, 1, 5), (70, 600, 3)])
@pytest.mark.parametrize("density", [0.0, 0.03, 1.0])
def test_leak_grad(T, B, N, density):
    rng = np.random.default_rng(T + B + N)
    alpha = math.exp(-0.1)
    f32alpha = float(np.float32(alpha))
    x = rng.standard_normal((T, B, N)).astype(np.float32)
    on_x, on_y = (rng.random((T, B, N)) < density for _ in range(2))
    g = rng.random((T, B, N)).astype(np.float32)
    gated = np.where(on_x, x.astype(np.float64) * g, 0.0)
    dx = torch.from_numpy(x).cuda()
    ex = torch.from_numpy(x[on_x]).cuda()
    csr_x, plain_x, csr_y = csr_of(on_x, g), csr_of(on_x), csr_of(on_y)
    # a step rounds its product and sum (and the gated entry) once, against the sum of absolute values
    for src, inp, ref in ((dx, None, x.astype(np.float64)), (ex, csr_x, gated), (ex, plain_x, np.where(on_x, x, 0.0))):
        want, bound = tokens.leak_grad(ref, f32alpha), tokens.leak_grad(np.abs(ref), f32alpha)
        tol = 2 * U * T * bound + 1e-37
        y = snn.leak_grad(src, alpha, (T, B, N), inp=inp)
        close(y, want, tol, "dense")
        e = snn.leak_grad(src, alpha, (T, B, N), inp=inp, out=csr_y)
        assert np.array_equal(host(e), host(y)[on_y])


def test_leak_grad_truncated():
    """Entries beyond a side's capacity are neither read nor written."""
    rng = np.random.default_rng(3)
    T, B, N, alpha = 40, 2, 70, 0.9
    on = rng.random((T, B, N)) < 0.1
    csr = csr_of(on)
    n = csr.capacity // 2
    x = rng.standard_normal(csr.capacity).astype(np.float32)
    csr.capacity = n
    dense = np.zeros((T, B, N))
    dense[tuple(a[:n] for a in np.nonzero(on))] = x[:n]
    y = snn.leak_grad(torch.from_numpy(x).cuda(), alpha, (T, B, N), inp=csr)
    close(y, tokens.leak_grad(dense, float(np.float32(alpha))), 1e-5, "dense")
    out = torch.full((len(x),), NAN, device="cuda")
    snn.leak_grad(torch.ones((T, B, N), device="cuda"), alpha, (T, B, N), out=csr, y=out)
    assert not out[:n].isnan().any() and out[n:].isnan().all()


@pytest.mark.parametrize("T,B,N", [(1, 2, 3), (2, 1, 64), (40, 3, 50), (33, 2, 256)])
def test_lif_forward_currents(T, B, N):
    """As the layer itself where its input is one spike a row: the same bits."""
    rng = np.random.default_rng(N)
    ids = ints(rng.integers(0, 20, (T, B)))
    W = torch.from_numpy(rng.standard_normal((20, N)).astype(np.float32)).cuda()
    S_in = torch.nn.functional.one_hot(ids.long(), 20).to(torch.uint8)
    outs = []
    for way in range(2):
        V, tr = (torch.empty((T, B, N), device="cuda") for _ in range(2))
        S = torch.empty((T, B, N), dtype=torch.uint8, device="cuda")
        bits = torch.zeros(snn.snn_active_bits_words(T, B, N), dtype=torch.int64, device="cuda")
        if way:
            snn.snn_lif_forward_traces(S_in, W, T, B, 20, N, 0.9, 1.0, 0.2, V, S, None, tr, 0.8, bits)
        else:
            if T > 1:
                snn.embed(W, ids[:-1], out=V[1:])
            snn.snn_lif_forward_currents(V, T, B, N, 0.9, 1.0, 0.2, S, tr, 0.8, bits)
        outs.append((V, S, tr, bits))
    assert all(torch.equal(p, q) for p, q in zip(*outs))
    V2 = outs[1][0].clone()
    if T > 1:
        snn.embed(W, ids[:-1], out=V2[1:])
    S2 = torch.empty((T, B, N), dtype=torch.uint8, device="cuda")
    snn.snn_lif_forward_currents(V2, T, B, N, 0.9, 1.0, 0.0, S2)
    assert torch.equal(V2, outs[1][0]) and torch.equal(S2, outs[1][1])


# ---------------------------------------------------------------- together, streams, graphs

def chain(E, ids, gamma, beta, W, targets):
    """Lookup, norm, loss and the gradients of all of them."""
    V, R, N = E.shape[0], ids.numel(), E.shape[1]
    e = snn.embed(E, ids, math.sqrt(N))
    y, mean, rstd = snn.layer_norm(e, gamma, beta)
    loss, row_loss, dy, dW = snn.linear_ce(y, W, targets)
    de, dgamma, dbeta = snn.layer_norm_grad(dy, e, gamma, mean, rstd)
    dE = snn.embed_grad(ids, de, V, math.sqrt(N))
    return loss, row_loss, dE, dgamma, dbeta, dW


def chain_inputs(dtype, seed, R=700, V=900, N=96, C=500):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    dt = DTYPES[dtype]
    return [r(V, N).mul(0.3).to(dt), torch.randint(-1, V, (R,), generator=g, device="cuda").to(torch.int32), 1 + 0.1 * r(N),
            0.1 * r(N), r(N, C).mul(0.2).to(dt), torch.randint(-1, C, (R,), generator=g, device="cuda").to(torch.int32)]


@pytest.mark.parametrize("dtype", DTYPES)
def test_chain(dtype):
    """A run of them as they are used, against autograd in 64 bits; differences along a direction."""
    args = chain_inputs(dtype, 1)
    loss, row_loss, dE, dgamma, dbeta, dW = chain(*args)
    leaves = [args[k].double().requires_grad_(True) for k in (0, 2, 3, 4)]
    ids, t = args[1].long(), args[5].long()

    def of(E, gamma, beta, W):
        e = E[ids.clamp_min(0)] * (ids >= 0)[:, None] * math.sqrt(96)
        z = torch.nn.functional.layer_norm(e, (96,), gamma, beta, 1e-5) @ W
        return torch.nn.functional.cross_entropy(z, t, ignore_index=-1)

    want = of(*leaves)
    u = ROUND[dtype][0]
    assert abs(float(loss) - float(want)) < 8 * u * 10 + 1e-5
    grads = torch.autograd.grad(want, leaves)
    for got, ref, name in zip((dE, dgamma, dbeta, dW), grads, ("dE", "dgamma", "dbeta", "dW")):
        # five roundings to the type on the way (lookup, norm, dz, dy, de), each of a random sign
        assert float((got.double() - ref).norm()) < (6 * u + 2e-5) * float(ref.norm()) + 1e-7, name
    if dtype == "f32":
        g = torch.Generator(device="cuda").manual_seed(9)
        d = [torch.randn(p.shape, generator=g, device="cuda", dtype=torch.float64) for p in leaves]
        with torch.no_grad():
            diff = float(of(*[p + 1e-5 * q for p, q in zip(leaves, d)]) - of(*[p - 1e-5 * q for p, q in zip(leaves, d)])) / 2e-5
        along = sum(float((p.double() * q).sum()) for p, q in zip((dE, dgamma, dbeta, dW), d))
        assert abs(diff - along) < 1e-4 * sum(float((p.double().norm() * q.norm())) for p, q in zip((dE, dgamma, dbeta, dW), d)) / 10


def test_streams_and_graphs():
    args = chain_inputs("bf16", 2)
    want = chain(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    E, ids, gamma, beta, W, t = args
    e = snn.embed(E, ids, math.sqrt(96), stream=side)
    y, mean, rstd = snn.layer_norm(e, gamma, beta, stream=side)
    loss, row_loss, dy, dW = snn.linear_ce(y, W, t, stream=side)
    de, dgamma, dbeta = snn.layer_norm_grad(dy, e, gamma, mean, rstd, stream=side)
    dE = snn.embed_grad(ids, de, E.shape[0], math.sqrt(96), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip((loss, row_loss, dE, dgamma, dbeta, dW), want))
    g = pipeline.Graphed(functools.partial(chain, *args))
    for k in range(3):
        other = chain_inputs("bf16", 3 + k)
        for p, q in zip(args, other):
            p.copy_(q)
        out = g()
        torch.cuda.synchronize()
        want = chain(*other)
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_python_refusals():
    x, W, t = torch.zeros((4, 8), device="cuda"), torch.zeros((8, 5), device="cuda"), ints([0, 1, 2, 3])
    with pytest.raises(ValueError):
        snn.linear_ce(x, torch.zeros((7, 5), device="cuda"), t)
    with pytest.raises(ValueError):
        snn.linear_ce(x, W.half(), t)
    with pytest.raises(ValueError):
        snn.linear_ce(x, W, ints([0, 1]))
    with pytest.raises(TypeError):
        snn.linear_ce(x, W, t.long())
    with pytest.raises(ValueError):
        snn.linear_ce(x, W, t.cpu())
    with pytest.raises(ValueError):
        snn.linear_ce(x, W.T.contiguous().T, t)
    with pytest.raises(ValueError):
        snn.embed_grad(t, x, 10, accumulate=True)
    with pytest.raises(ValueError):
        snn.embed_grad(t, x, 10, dE=torch.zeros((9, 8), device="cuda"))
    with pytest.raises(ValueError):
        snn.embed(W, ints([0]), out=torch.zeros((1, 6), device="cuda"))
    with pytest.raises(TypeError):
        snn.embed(W, t.long())
    with pytest.raises(snn.SnnError):
        snn.layer_norm(x, eps=-1.0)
    with pytest.raises(ValueError):
        snn.layer_norm(x, gamma=torch.zeros(7, device="cuda"))
    with pytest.raises(snn.SnnError):
        snn.leak_grad(torch.zeros((2, 2, 2), device="cuda"), 1.5, (2, 2, 2))
    with pytest.raises(ValueError):
        snn.leak_grad(torch.zeros((2, 2, 2), device="cuda"), 0.5, (2, 2, 3))
