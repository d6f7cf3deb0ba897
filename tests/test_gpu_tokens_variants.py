"""Every way that the operators on token sequences choose by their sizes, at small sizes on both sides of its line: both tiles
of 16-bit cross entropy with W read in place and copied, all class counts of the two ways of few classes, rows of classes
by wavefronts, by blocks and re-read, all shapes of layer norm. Against 64 bits on the device, rows without a target NaN, a
poisoned workspace."""
import math

import pytest
import torch

import test_gpu_tokens as base
from paper_2105_08810_amd import snn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def within(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(0).max())} of the tolerance"


def check(R, H, C, dtype, ld_x=0, ld_w=0, lead=0, dead=0.1, weighted=False, seed=0):
    """linear_ce on R x H x C; rows of x and W in ld_x and ld_w more elements, `lead` past an aligned address."""
    dt = base.DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(R + H + C + seed)

    def rows(z, more):
        full = torch.full((z.shape[0] * (z.shape[1] + more) + lead,), math.nan, dtype=dt, device="cuda")
        view = full[lead:].view(z.shape[0], z.shape[1] + more)[:, :z.shape[1]]
        view.copy_(z)
        return view

    x = rows(torch.randn((R, H), generator=g, device="cuda"), ld_x)
    W = rows(torch.randn((H, C), generator=g, device="cuda") * (2.0 / math.sqrt(H)), ld_w)
    t = torch.randint(0, C, (R,), generator=g, device="cuda").to(torch.int32)
    t[torch.rand(R, generator=g, device="cuda") < dead] = -1
    t[0] = C - 1
    w = None
    if weighted:
        w = torch.rand(R, generator=g, device="cuda")
        w[torch.rand(R, generator=g, device="cuda") < 0.1] = 0.0
        w[0] = 1.0
    live = t >= 0 if w is None else (t >= 0) & (w != 0)
    X = x.double() * live[:, None]
    x[~live] = math.nan
    ws, behind = base.poisoned(snn.snn_linear_ce_workspace(dt, R, H, C, True))
    loss, row_loss, dx, dW = snn.linear_ce(x, W, t, w, ws=ws)
    assert bool((behind == 255).all())

    W64 = W.double()
    k = torch.where(live, 1.0 / live.sum() if w is None else w.double(), 0.0)
    at = t.clamp_min(0).long()[:, None]
    z = X @ W64
    bound = (X.abs() @ W64.abs()).amax(1, keepdim=True)
    others = z.scatter(1, at, -math.inf)
    zt = z.gather(1, at)
    m = torch.maximum(others.amax(1, keepdim=True), zt)
    rest = torch.exp(others - m).sum(1, keepdim=True)
    s = rest + torch.exp(zt - m)
    row = ((m - zt) + torch.log(s))[:, 0]
    p = torch.exp(others - m) / s
    p.scatter_(1, at, -rest / s)
    dz = p * k[:, None]
    # z: H products summed in float32, steps rounded towards zero (2 U each), as are three-part products; an exponential twice
    # that, a sum of C of them and roundings of arguments below 60
    ez = 2 * (H + 4) * U * bound
    rel = 2 * ez + (C / 64 + 100) * U
    tol = (2 * ez + (C / 64 + 40) * U + 8 * U * (1 + row[:, None]))[:, 0]
    assert not bool(row_loss[~live].any()) and not bool(dx[~live].any())
    within(row_loss[live], row[live], tol[live], "row_loss")
    within(loss[0], (k * row).sum(), (k * tol).sum() + 4 * U * (k * row).sum(), "loss")
    u, least = base.ROUND[dtype]
    narrow = dtype != "f32" and not (C <= 128 and R <= 4096)  # dz in the type
    e = dz.abs() * (rel + (u if narrow else 0.0))
    if narrow:  # below the type's numbers, as a share of the largest weight
        e += live[:, None] * k.max() * (2.0 ** -126 if dtype == "bf16" else 2.0 ** -40)
    tol = e @ W64.abs().T + 2 * (C + 4) * U * (dz.abs() @ W64.abs().T)
    want = dz @ W64.T
    within(dx, want, tol + u * (want.abs() + tol) + least, "dx")
    tol = X.abs().T @ e + 2 * (R + 4) * U * (X.abs().T @ dz.abs())
    want = X.T @ dz
    within(dW, want, tol + u * (want.abs() + tol) + least, "dW")
    again = snn.linear_ce(x, W, t, w)
    assert all(torch.equal(p, q) for p, q in zip(again, (loss, row_loss, dx, dW)))


# H beyond 128 and 512 tiles of 256 x 256: the large tile; one more row, hidden value and class than whole tiles
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("R,H,C,ld_x,ld_w,lead", [
    (4096, 256, 8192, 0, 0, 0), (4096, 256, 8192, 0, 8, 8), (4096, 256, 8192, 3, 5, 1), (4100, 192, 9001, 0, 0, 0),
    (256, 256, 131072, 0, 0, 0), (257, 257, 131073, 0, 3, 0), (255, 129, 130817, 1, 0, 0)])
@pytest.mark.parametrize("weighted", [False, True])
def test_large_tile(dtype, R, H, C, ld_x, ld_w, lead, weighted):
    check(R, H, C, dtype, ld_x, ld_w, lead, weighted=weighted)


# W in place at the small tile: whole tiles, rows at multiples of 16 bytes; and the same copied
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("R,H,C", [(300, 128, 256), (130, 256, 1024), (1, 128, 384), (4200, 128, 128), (4200, 384, 100)])
@pytest.mark.parametrize("ld_w,lead", [(0, 0), (8, 0), (8, 8), (8, 1), (4, 0)])
def test_small_tile(dtype, R, H, C, ld_w, lead):
    check(R, H, C, dtype, 0, ld_w, lead)


# few classes of many float32 rows: 16 and, from 65409 rows on 256 compute units, 32 rows a wavefront, every number of class
# tiles, hidden sizes that are multiples of 8 and not
@pytest.mark.parametrize("R", [5000, 65409, 70001])
@pytest.mark.parametrize("H", [8, 33])
@pytest.mark.parametrize("C", [7, 16, 30, 50, 101, 112, 120, 128])
def test_few_classes(R, H, C):
    check(R, H, C, "f32", 0, 0, 0, weighted=(C + R) % 2 == 0)


# rows of float32 classes in one wavefront, in blocks of every depth, and beyond what a block keeps; logits in K slices
@pytest.mark.parametrize("R,H,C", [(5, 8, 129), (5, 8, 257), (5, 8, 600), (5, 8, 1025), (3, 8, 5000), (3, 8, 9000),
                                   (3, 8, 20000), (3, 8, 32768), (3, 8, 32769), (3, 8, 40000), (20, 2048, 200),
                                   (20, 2048, 9000), (7, 3000, 17000), (600, 8, 9000)])
@pytest.mark.parametrize("ld_w,lead", [(0, 0), (3, 1)])
def test_rows_of_classes(R, H, C, ld_w, lead):
    check(R, H, C, "f32", 0, ld_w, lead, dead=0.2, weighted=lead == 1)


# float32 in pieces, whose first classes are not the target's
@pytest.mark.parametrize("R,H,C", [(3000, 8, 50001), (520, 4, 260001)])
def test_pieces(R, H, C):
    check(R, H, C, "f32")


# 16 bits in pieces, at either tile
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("R,H,C", [(4100, 16, 66000), (2100, 130, 131000)])
def test_pieces_in_16_bits(dtype, R, H, C):
    check(R, H, C, dtype)


# a row in every number of vectors and lanes
@pytest.mark.parametrize("dtype,N", [("f32", n) for n in (60, 65, 250, 300, 500, 513, 768, 769, 1020, 1030, 1280, 1281, 1500,
                                                          1537, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385)]
                         + [(d, n) for d in ("bf16", "f16") for n in (120, 129, 500, 513, 1024, 1025, 2049, 3073, 4096, 4097,
                                                                       8192, 8193, 16384, 16385, 32768, 32769)])
def test_widths_of_norm(dtype, N):
    base.test_layer_norm(dtype, dtype, 3, N, "both", 0, 0)
    base.test_layer_norm(dtype, dtype, 2, N, "gamma", 3, 1)


# rows on both sides of the line between one block's places and the scan's
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("R", [8192, 8193, 20000, 32769])
@pytest.mark.parametrize("weighted", [False, True])
def test_places(dtype, R, weighted):
    check(R, 8, 300, dtype, dead=0.3, weighted=weighted)
