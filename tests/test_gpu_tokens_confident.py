"""Cross entropy of linear logits for rows that are nearly certain of their target, with an offset common to all classes,
which softmax ignores: the gradient by the target's logit is minus the others' share, however large the logits are."""
import math

import pytest
import torch

from paper_2105_08810_amd import snn

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a step of a result's type, and of its smallest numbers
ROUND = {"f32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}
U = 2.0 ** -24


def case(R, K, H, C, dtype, offset, margin, seed):
    """Rows of K kinds: z = offset + W[1 + kind], all of few bits, so that logits are exact in float32 in any order of
    sums. The target lies `margin` above the largest of the others."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.arange(R, device="cuda") % K
    x = torch.zeros((R, H), device="cuda")
    x[:, 0] = 1.0
    x[torch.arange(R, device="cuda"), 1 + kind] = 1.0
    W = torch.zeros((H, C), device="cuda")
    W[0] = offset
    W[1:1 + K] = torch.randint(-32, 1, (K, C), generator=g, device="cuda") / 16.0
    target = torch.randint(0, C, (K,), generator=g, device="cuda")
    W[1 + torch.arange(K, device="cuda"), target] = margin
    x, W = x.to(DTYPES[dtype]), W.to(DTYPES[dtype])
    z = W[1:1 + K].double()
    others = z.clone()
    others[torch.arange(K, device="cuda"), target] = -math.inf
    e = torch.exp(others - margin)
    rest = e.sum(1, keepdim=True)
    share = e / (1.0 + rest)
    share[torch.arange(K, device="cuda"), target] = -(rest / (1.0 + rest))[:, 0]
    return x, W, target[kind].to(torch.int32), kind, share, torch.log1p(rest)[:, 0]


CASES = [
    ("f32", 48, 48, 50, 10), ("f32", 48, 48, 50, 100), ("f32", 4400, 44, 45, 10), ("f32", 4400, 44, 45, 100),
    ("f32", 66000, 44, 45, 100), ("f32", 96, 48, 50, 300), ("f32", 96, 48, 50, 1000), ("f32", 96, 48, 50, 2000),
    ("f32", 24, 8, 9, 20000), ("f32", 24, 8, 9, 40000), ("f32", 3000, 8, 9, 47001),
    ("bf16", 48, 48, 50, 10), ("bf16", 48, 48, 50, 100), ("bf16", 96, 48, 50, 300), ("bf16", 4400, 44, 45, 100),
    ("bf16", 1025, 41, 130, 32800), ("f16", 48, 48, 50, 10), ("f16", 48, 48, 50, 100), ("f16", 96, 48, 50, 300),
    ("f16", 4400, 44, 45, 100), ("f16", 1025, 41, 130, 32800),
]


@pytest.mark.parametrize("dtype,R,K,H,C", CASES)
@pytest.mark.parametrize("offset", [0.0, 16.0, 256.0])
@pytest.mark.parametrize("weighted", [False, True])
def test_confident_rows(dtype, R, K, H, C, offset, weighted):
    margin = float(round(math.log(C))) + 6.0
    x, W, t, kind, share, row = case(R, K, H, C, dtype, offset, margin, R + C)
    weight = torch.ones(R, device="cuda") if weighted else None
    loss, row_loss, dx, dW = snn.linear_ce(x, W, t, weight)
    w = 1.0 if weighted else 1.0 / R
    # an exponential is two roundings off, in the 16-bit kernels also its argument's, |z - largest| log2(e) at most 28 and
    # formed with two roundings; the sum of the others C / 64 + 6, a share's quotient and product 4
    rel = (2 + 2 * 28 + C / 64 + 6 + 4) * U
    got = row_loss.double()
    assert float(((got - row[kind]).abs() / row[kind]).max()) < rel + 4 * U  # the logarithm, and its argument's share
    assert abs(float(loss) - w * float(row[kind].sum())) < (rel + 8 * U) * w * float(row[kind].sum())
    # dW of a kind's row is the sum of its rows' equal dz. dz is rounded to a 16-bit type once, float16's below 2^-14 of the
    # largest weight (raised by 2^15) to steps of 2^-39; the sum of n equal terms, its products' parts and its slices n + 8
    n = torch.bincount(kind, minlength=K).double()[:, None]
    u, least = ROUND[dtype]
    one, small = {"f32": (0.0, 0.0), "bf16": (u, 2.0 ** -126), "f16": (u, 2.0 ** -40)}[dtype]
    if R <= 4096 and C <= 128:  # products in float32
        one = small = 0.0
    want = w * n * share
    tol = want.abs() * (rel + one + 2 * (n + 8) * U) + w * n * small
    tol = tol + u * (want.abs() + tol) + least
    bad = (dW[1:1 + K].double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float(((dW[1:1 + K].double() - want).abs() / tol).max()))
