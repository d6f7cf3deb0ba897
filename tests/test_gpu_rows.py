"""The operators on rows of logits against the float64 oracle: every type, lengths from one class to long rows, padded and
misaligned rows, ties, masked classes, empty rows, infinities and NaN."""
import functools
import math

import numpy as np
import pytest
import torch

from oracle import rows
from paper_2105_08810_amd import snn

pytestmark = pytest.mark.gpu



@pytest.fixture(autouse=True)
def _quiet():
    """Differences of infinities, which the masks beside them leave out."""
    with np.errstate(invalid="ignore"):
        yield


INF = math.inf
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# relative rounding of a result to its type, and the spacing of its smallest numbers
ROUND = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 2.0 ** -133), "f16": (2.0 ** -11, 2.0 ** -25)}
U = 2.0 ** -24


def _rows(z, dtype, ld=None, lead=0):
    """z [R, C] on the device as rows of dtype in rows of ld elements, `lead` elements past an aligned address; the
    elements around hold NaN, which nothing may read as a class."""
    R, C = z.shape
    ld = C if ld is None else ld
    full = torch.full((R * ld + lead,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = full[lead:].view(R, ld)[:, :C]
    view.copy_(torch.from_numpy(np.ascontiguousarray(z)).cuda())
    return view


def _values(view):
    return view.float().cpu().numpy()


def _logits(rng, R, C, kind):
    z = (rng.standard_normal((R, C)) * 2.5).astype(np.float32)
    if kind == "ties":
        z = np.round(z)
    if kind == "equal":
        z[:] = 0.75
    if kind == "zeros":  # both zeros are one value
        z = np.where(rng.random((R, C)) < 0.5, np.float32(0.0), np.float32(-0.0))
    if kind == "masked":
        z[rng.random((R, C)) < 0.4] = -INF
        z[0, :] = -INF
        if R > 1:
            z[1, :] = -INF
            z[1, C // 2] = -3.0
    if kind == "lowest":  # masks of the type's lowest value
        z[rng.random((R, C)) < 0.4] = -60000.0
        z[0, :] = -60000.0
    if kind == "nan":
        z[rng.random((R, C)) < 0.2] = np.nan
        z[0, :] = np.nan
        z[0, C - 1] = 1.0
    if kind == "inf":
        z[:, C // 3] = INF
        if R > 1:
            z[1, C - 1] = INF
    if kind == "wide":  # values far apart, and close together far away
        z = (z * 10.0 ** rng.integers(-6, 4, (R, C))).astype(np.float32)
    if kind == "peak":
        z[np.arange(R), rng.integers(0, C, R)] = 40.0
    return z


def _adds(C):
    """Float32 additions one after another in a row's sum, at most: a thread's share, then a tree."""
    return C / 1024 + 64 + 22


# (R, C, ld, lead): one class to more than any tile, lengths beside powers of two, padded and misaligned rows
SHAPES = [(1, 1, None, 0), (3, 1, 4, 1), (5, 2, None, 0), (300, 3, None, 0), (7, 10, 10, 3), (65, 20, None, 0),
          (2, 63, None, 0), (9, 64, 65, 0), (33, 65, 67, 5), (130, 100, 100, 0), (4, 127, None, 1), (3, 128, 131, 7),
          (5, 129, None, 0), (6, 255, 256, 0), (3, 256, None, 0), (5, 257, 300, 2), (4, 511, None, 0), (3, 513, None, 6),
          (3, 1000, None, 0), (2, 1024, None, 0), (3, 1025, 1031, 3), (2, 2047, None, 0), (3, 4096, 4100, 0),
          (2, 4099, None, 1), (2, 8193, None, 0), (2, 16384, None, 0), (3, 16387, 16400, 5), (2, 32771, None, 0),
          (1, 65536, None, 0), (2, 65601, None, 3), (1, 131072, None, 0), (1, 140003, None, 1)]
KINDS = ["normal", "ties", "equal", "zeros", "masked", "lowest", "nan", "inf", "wide", "peak"]


def _kinds(i):
    """Two kinds for each shape, so that all come up at several lengths."""
    return [KINDS[i % len(KINDS)], KINDS[(3 * i + 4) % len(KINDS)]]


CASES = [(s, k, d) for i, s in enumerate(SHAPES) for j, k in enumerate(_kinds(i))
         for d in (("f32", "bf16", "f16")[(i + j) % 3], "f32")]
CASES = list(dict.fromkeys(CASES))


def _id(v):
    return "-".join(map(str, v)) if isinstance(v, tuple) else str(v)


# ---------------------------------------------------------------- records

def _check_top(z, view, K, tau):
    ids, vals, lse = snn.readout_top(view, K, tau)
    i, v, l = rows.top(z, K, tau)
    assert np.array_equal(ids.cpu().numpy(), i)
    assert np.array_equal(vals.cpu().numpy().astype(np.float64), v)
    got = lse.cpu().numpy().astype(np.float64)
    fine = np.isfinite(l)
    assert np.array_equal(got[~fine], l[~fine])
    # m/tau (two roundings), log (a few ulp of a number below log C), the last addition; the exponents' error of
    # |x - m|/tau 2U only counts where exp is not small: x e^-x < 0.4; then the sum's additions
    m = np.abs(np.where(np.isfinite(z), z, 0)).max(1) / tau
    tol = U * (4 * m + 8 * (1 + math.log(z.shape[1])) + _adds(z.shape[1]))
    assert (np.abs(got - l)[fine] <= tol[fine]).all()


@pytest.mark.parametrize("shape,kind,dtype", CASES, ids=_id)
def test_top(shape, kind, dtype):
    R, C, ld, lead = shape
    rng = np.random.default_rng(R * 7 + C)
    view = _rows(_logits(rng, R, C, kind), dtype, ld, lead)
    z = _values(view)
    for K in sorted({1, min(C, 5), min(C, 64), min(C, 300)}):
        _check_top(z, view, K, 1.7)


@pytest.mark.parametrize("C,K", [(1024, 1024), (1025, 1024), (20000, 1024), (70000, 777), (700, 700)])
@pytest.mark.parametrize("kind", ["normal", "ties", "masked"])
def test_top_long_records(C, K, kind):
    rng = np.random.default_rng(C + K)
    view = _rows(_logits(rng, 3, C, kind), "f32")
    _check_top(_values(view), view, K, 0.5)


def test_top_of_a_readout():
    V = torch.randn((11, 5, 37), device="cuda")
    ids, vals, lse = snn.readout_top(V, 4, 2.0)
    assert ids.shape == (11, 5, 4) and vals.shape == (11, 5, 4) and lse.shape == (11, 5)
    i, v, l = rows.top(V.view(55, 37).cpu().numpy(), 4, 2.0)
    assert np.array_equal(ids.view(55, 4).cpu().numpy(), i) and np.array_equal(vals.view(55, 4).cpu().numpy(), v)


# ---------------------------------------------------------------- distillation

def _record(rng, z, K, tau, kind):
    t = (0.7 * np.where(np.isfinite(z), z, 0.0) + rng.standard_normal(z.shape)).astype(np.float32)
    ids, vals, lse = rows.top(t, K, tau)
    ids, vals, lse = ids.astype(np.int32), vals.astype(np.float32), lse.astype(np.float32)
    order = rng.permutation(K)  # the entries may come in any order
    ids, vals = np.ascontiguousarray(ids[:, order]), np.ascontiguousarray(vals[:, order])
    if kind == "holes":  # ids outside the classes, whole records of them, entries of no probability
        ids[rng.random(ids.shape) < 0.3] = -1
        ids[0, :] = z.shape[1] + 5
        vals[rng.random(ids.shape) < 0.1] = -INF
    return ids, vals, lse


def _check_distill(view, ids, vals, lse, tau, weight, dtype, start=None, ld_grad=None):
    z = _values(view)
    R, C = z.shape
    K = ids.shape[1]
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    kw = {}
    if start is not None:
        kw = dict(grad=start, accumulate=True)
        before = _values(start).astype(np.float64)
    loss, row_loss, grad = snn.readout_distill(view, dev(ids), dev(vals), dev(lse), tau, dev(weight), **kw)
    with np.errstate(all="ignore"):
        lo, rl, g, env, share = rows.distill(z.astype(np.float64), ids, vals, lse, tau, weight)
    got_l, got_r, got_g = float(loss), row_loss.cpu().numpy().astype(np.float64), _values(grad).astype(np.float64)
    # The exponents of q are differences of numbers of size A, formed in float32 with a few roundings; those of p
    # likewise from vals/tau and lse. p_t = 1 - sum p has the absolute error of its terms.
    w = np.full(R, 1.0 / R) if weight is None else weight.astype(np.float64)
    fin = lambda a: np.where(np.isfinite(a), a, 0.0)  # noqa: E731
    A = np.abs(fin(z)).max(1) / tau + np.abs(fin(vals)).max(1) / tau + 1
    rel = U * (16 + _adds(C) + K / 64 + 6 * A)
    d_t = rel if lse is not None else np.zeros(R)
    big = np.array([sum(abs(v) for v in _terms(z[r], ids[r], vals[r], None if lse is None else lse[r], tau))
                    for r in range(R)])
    tol_r = rel * (1 + big) + d_t * (2 + A)
    fine = np.isfinite(rl)
    assert np.array_equal(np.isnan(got_r), np.isnan(rl)) and np.array_equal(got_r[~fine & ~np.isnan(rl)], rl[~fine & ~np.isnan(rl)])
    assert (np.abs(got_r - rl)[fine] <= tol_r[fine]).all()
    if fine.all():
        assert abs(got_l - lo) <= (np.abs(w) * tol_r).sum() + U * abs(lo)
    want = g if start is None else g + np.where(w[:, None] != 0, before, before)
    r_out, tiny = ROUND[dtype]
    whole = np.isfinite(want)
    assert np.array_equal(np.isnan(got_g), np.isnan(want))
    # the error of p_t goes to the other classes by their share q / q_t
    tol = rel[:, None] * env + (np.abs(w) / tau * d_t)[:, None] * share * 4
    extra = 0.0 if start is None else 2 * U * np.abs(want)
    tol = tol + extra + r_out * (np.abs(want) + tol) * 1.01 + tiny + 2.0 ** -126
    bad = ~(np.abs(got_g - want) <= tol) & whole
    assert not bad.any(), (np.argwhere(bad)[:5], got_g[bad][:5], want[bad][:5], tol[bad][:5])


def _terms(z, ids, vals, lse, tau):
    """The loss's terms p log p and p log q of a row."""
    C = len(z)
    z = z.astype(np.float64) / tau
    if not (z > -INF).any() or np.isnan(z).any():
        return [0.0]
    logq = z - rows.log_sum_exp(z)
    ok = (ids >= 0) & (ids < C)
    v = vals[ok].astype(np.float64) / tau
    if not len(v) or np.max(v) == -INF:
        return [0.0]
    logp = v - (rows.log_sum_exp(v) if lse is None else float(lse))
    out = []
    for lp, lq in zip(logp, logq[ids[ok]]):
        if lp > -INF and np.isfinite(lq):
            out += [math.exp(lp) * lp, math.exp(lp) * lq]
    return out or [0.0]


@pytest.mark.parametrize("shape,kind,dtype", CASES, ids=_id)
def test_distill(shape, kind, dtype):
    R, C, ld, lead = shape
    rng = np.random.default_rng(R * 11 + C)
    view = _rows(_logits(rng, R, C, kind), dtype, ld, lead)
    z = _values(view)
    weight = rng.random(R).astype(np.float32)
    weight[::3] = 0.0
    for n, K in enumerate(sorted({1, min(C, 7), min(C, 130)})):
        tau = (1.0, 1.5, 4.0)[n]
        rec = _record(rng, z, K, tau, "holes" if n == 1 else "")
        _check_distill(view, rec[0], rec[1], rec[2] if n != 1 else None, tau, weight if n != 0 else None, dtype)
        _check_distill(view, rec[0], rec[1], rec[2] if n == 1 else None, tau, None if n != 0 else weight, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,ld,lead", [(5, 10, 13, 1), (3, 700, 701, 0), (2, 5000, 5003, 2), (2, 40000, None, 0)])
def test_distill_adds_to_a_gradient(dtype, R, C, ld, lead):
    rng = np.random.default_rng(C)
    view = _rows(rng.standard_normal((R, C)).astype(np.float32), dtype, ld, lead)
    start = _rows(rng.standard_normal((R, C)).astype(np.float32) * 1e-2, dtype, ld and ld + 1, lead + 1)
    weight = np.linspace(0, 1, R).astype(np.float32)
    rec = _record(rng, _values(view), 6, 2.0, "")
    _check_distill(view, *rec, 2.0, weight, dtype, start=start)


def test_distill_loss_alone_and_padding_untouched():
    rng = np.random.default_rng(3)
    z = rng.standard_normal((6, 50)).astype(np.float32)
    view = _rows(z, "f32", 56, 0)
    ids, vals, lse = (torch.from_numpy(a).cuda() for a in _record(rng, z, 4, 1.0, ""))
    a = snn.readout_distill(view, ids, vals, lse, 1.0, want_grad=False)
    full = torch.full((6, 60), 7.0, device="cuda")
    b = snn.readout_distill(view, ids, vals, lse, 1.0, grad=full[:, :50])
    assert a[2] is None and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool((full[:, 50:] == 7.0).all()) and not bool((full[:, :50] == 7.0).any())


def test_distill_rows_without_weight_are_not_read():
    z = torch.randn((4, 30), device="cuda")
    z[1] = float("nan")
    ids = torch.tensor([[1, 5], [2, 3], [0, 29], [7, -1]], dtype=torch.int32, device="cuda")
    vals = torch.tensor([[1.0, 0.5], [float("nan"), INF], [0.0, 2.0], [1.0, 1.0]], device="cuda")
    w = torch.tensor([0.5, 0.0, 0.25, 0.25], device="cuda")
    loss, row_loss, grad = snn.readout_distill(z, ids, vals, None, 1.0, w)
    assert bool(torch.isfinite(loss).all()) and float(row_loss[1]) == 0.0
    assert bool((grad[1] == 0).all()) and bool(torch.isfinite(grad).all())


def test_distill_not_finite_rows():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((5, 9)).astype(np.float32)
    z[1, 4] = np.nan
    z[2, 4] = INF
    z[3, :] = -INF
    z[4, 2] = -INF
    ids = np.tile(np.array([[4, 2]], np.int32), (5, 1))
    vals = np.tile(np.array([[1.0, 0.0]], np.float32), (5, 1))
    loss, row_loss, grad = snn.readout_distill(torch.from_numpy(z).cuda(), torch.from_numpy(ids).cuda(),
                                               torch.from_numpy(vals).cuda(), None, 1.0)
    l, g = row_loss.cpu().numpy(), grad.cpu().numpy()
    p = np.array([math.e, 1.0]) / (1 + math.e)
    assert np.isfinite(l[0]) and np.isfinite(g[0]).all()
    assert np.isnan(l[1]) and np.isnan(g[1]).all() and np.isnan(l[2]) and np.isnan(g[2]).all()
    assert l[3] == INF and np.allclose(g[3, [4, 2]], -p / 5, atol=1e-7) and g[3].astype(bool).sum() == 2
    assert l[4] == INF and np.isfinite(g[4]).all() and abs(g[4, 2] + p[1] / 5) < 1e-7


def test_distill_gradient_is_the_differences():
    """Along a direction d the losses of z + h d and z - h d differ by 2 h g.d: float32 losses of size 1 to 10 are
    within 100 U of themselves, the third derivative along d is below |d|^3 = 1."""
    rng = np.random.default_rng(8)
    for C, K in ((10, 3), (300, 20), (5000, 50)):
        z = rng.standard_normal((1, C)).astype(np.float32)
        rec = [torch.from_numpy(a).cuda() for a in _record(rng, z, K, 1.0, "")]
        d = rng.standard_normal((1, C))
        d = (d / np.linalg.norm(d)).astype(np.float32)
        h = 0.05
        f = lambda x: float(snn.readout_distill(torch.from_numpy(x.astype(np.float32)).cuda(), *rec, 1.0)[0])  # noqa: E731
        g = snn.readout_distill(torch.from_numpy(z).cuda(), *rec, 1.0)[2].cpu().numpy()
        diff = (f(z + h * d) - f(z - h * d)) / (2 * h)
        assert abs(diff - float((g.astype(np.float64) * d).sum())) <= h * h / 6 + 1000 * U / h


# ---------------------------------------------------------------- drawing

def _e(z, temperature):
    """exp((z - max) / temperature) in float32 as torch forms it on the device."""
    x = torch.from_numpy(np.where(np.isnan(z), -INF, z)).cuda()
    m = x.amax(1, keepdim=True)
    t = torch.from_numpy(temperature).cuda()[:, None]
    inv = torch.where(t > 0, 1.0 / t, torch.full_like(t, INF))
    return torch.exp(torch.where(x == m, torch.zeros_like(x), (x - m) * inv)).cpu().numpy()


def _check_sample(view, u, temperature, top_k, top_p, min_p):
    z = _values(view)
    R, C = z.shape
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    cls, logp, kept = (t.cpu().numpy() for t in snn.readout_sample(view, dev(u), dev(temperature), dev(top_k),
                                                                   dev(top_p), dev(min_p)))
    tt = np.ones(R, np.float32) if temperature is None else temperature
    e = _e(z, tt)
    for r in range(R):
        j, n, total, own = rows.sample_row(z[r], e[r], u[r], 0 if top_k is None else int(top_k[r]),
                                           1.0 if top_p is None else top_p[r], 0.0 if min_p is None else min_p[r],
                                           not tt[r] > 0)
        assert (cls[r], kept[r]) == (j, n), (r, tt[r], top_k is None or top_k[r], top_p is None or top_p[r])
        if j < 0:
            assert logp[r] == -INF
        else:  # a quotient of the logits' difference, a log below 22, one difference; a weight is within 2^-32 of its e
            want = math.log(float(e[r, j]) * rows.UNIT / total)
            assert abs(logp[r] - want) <= U * 8 * (24 + abs(want))


def _settings(rng, R, C):
    temperature = (0.3 + 1.5 * rng.random(R)).astype(np.float32)
    top_k = rng.integers(0, min(C, 60) + 1, R).astype(np.int32)
    top_p = (0.3 + 0.8 * rng.random(R)).astype(np.float32)
    min_p = np.where(rng.random(R) < 0.5, 0.0, 0.2 * rng.random(R)).astype(np.float32)
    return temperature, top_k, top_p, min_p


@pytest.mark.parametrize("shape,kind,dtype", CASES, ids=_id)
def test_sample(shape, kind, dtype):
    R, C, ld, lead = shape
    rng = np.random.default_rng(R * 13 + C)
    view = _rows(_logits(rng, R, C, kind), dtype, ld, lead)
    t, k, p, m = _settings(rng, R, C)
    for _ in range(2 if C > 20000 else 4):
        u = rng.random(R).astype(np.float32)
        _check_sample(view, u, None, None, None, None)
        _check_sample(view, u, t, k, p, m)
        _check_sample(view, u, t, None, p, None)
        _check_sample(view, u, None, k, None, None)
        if C <= 20000:
            _check_sample(view, u, t, None, None, m)
            _check_sample(view, u, t, k, p, None)


@pytest.mark.parametrize("C", [1, 2, 40, 300, 3000, 30000])
def test_sample_ends_of_the_settings(C):
    rng = np.random.default_rng(C)
    ends = [(0.0, 0, 1.0, 0.0), (-1.0, 5, 0.5, 0.1), (float("nan"), 0, 1.0, 0.0), (1.0, 1, 1.0, 0.0), (1.0, -3, 0.0, 0.0),
            (1.0, C + 7, -1.0, 0.0), (1.0, 0, 2.0, 1.0), (1.0, 0, 1.0, 5.0), (1.0, 0, 1.0, -1.0), (1.0, C, 1.0, 0.0),
            (1e-6, 0, 1.0, 0.0), (1e4, 0, 0.9, 0.0), (1.0, 0, 1e-9, 0.0), (1.0, 0, 0.99999994, 0.0), (1e-38, 0, 1.0, 0.0)]
    R = len(ends)
    z = _logits(rng, R, C, "normal")
    s = np.array(ends, np.float32)
    for u in (0.0, 0.37, float(np.float32(1 - 2 ** -24))):
        _check_sample(_rows(z, "f32"), np.full(R, u, np.float32), s[:, 0].copy(), s[:, 1].astype(np.int32),
                      s[:, 2].copy(), s[:, 3].copy())
    # uniforms outside [0, 1) are its ends; infinite temperatures make all finite classes alike
    view = _rows(z, "f32")
    dev = lambda v: torch.full((R,), v, device="cuda")  # noqa: E731
    for u, ref in ((-1.0, 0.0), (float("nan"), 0.0), (1.0, 1 - 2.0 ** -24), (7.0, 1 - 2.0 ** -24)):
        a, b = snn.readout_sample(view, dev(u)), snn.readout_sample(view, dev(ref))
        if u < 1.0 or u != u:
            assert torch.equal(a[0], b[0])
        else:
            assert bool((a[0] >= b[0]).all())
    cls, logp, kept = snn.readout_sample(view, dev(0.5), dev(INF))
    assert bool((kept == C).all()) and bool((cls == C // 2).all())
    assert float((logp + math.log(C)).abs().max()) < 1e-5


def test_sample_frequencies():
    """40000 draws of one row: a frequency is within five standard deviations of its probability in 64 bits."""
    rng = np.random.default_rng(1)
    z = (rng.standard_normal(12) * 1.5).astype(np.float32)
    n = 40000
    u = ((np.arange(n) + rng.random(n)) / n).astype(np.float32).clip(0, 1 - 2.0 ** -24)
    view = torch.from_numpy(np.tile(z, (n, 1))).cuda()
    t = torch.full((n,), 0.8, device="cuda")
    k = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    cls, logp, kept = snn.readout_sample(view, torch.from_numpy(u).cuda(), t, k)
    p = np.exp(z.astype(np.float64) / np.float32(0.8))
    p[rows.order(z)[9:]] = 0
    p /= p.sum()
    f = np.bincount(cls.cpu().numpy(), minlength=12) / n
    assert (np.abs(f - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()
    assert np.abs(logp.cpu().numpy() - np.log(p[cls.cpu().numpy()])).max() < 1e-5
    assert bool((kept == 9).all())


# ---------------------------------------------------------------- long offsets, streams, graphs, refusals

def test_offsets_past_32_bits():
    """Rows that begin beyond 2^32 elements (8.6 GB of bfloat16)."""
    C, ld, R = 1000, (1 << 31) + 11, 3
    full = torch.empty(R * ld, dtype=torch.bfloat16, device="cuda")
    view = full.view(R, ld)[:, :C]
    z = torch.randn((R, C), device="cuda").to(torch.bfloat16)
    view.copy_(z)
    # rows at other addresses than z's sum their float32 terms in another order: a row's log-sum-exp, of size below 16,
    # agrees within the rounding of its 1000 terms
    a, b = snn.readout_top(view, 5), snn.readout_top(z, 5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and float((a[2] - b[2]).abs().max()) < U * (_adds(C) + 16)
    u = torch.rand(R, device="cuda")
    for a, b in zip(snn.readout_sample(view, u), snn.readout_sample(z, u)):
        assert torch.equal(a, b)
    ids, vals, lse = snn.readout_top(torch.randn((R, C), device="cuda"), 5)
    a = snn.readout_distill(view, ids, vals, lse, grad=view.clone(memory_format=torch.contiguous_format))
    b = snn.readout_distill(z, ids, vals, lse)
    tol = U * (_adds(C) + 64)
    assert float((a[0] - b[0]).abs()) < tol * 16
    near = lambda x, y: bool(((x.float() - y.float()).abs() <= 2.0 ** -7 * y.float().abs() + tol).all())  # noqa: E731
    assert near(a[2], b[2])  # one step of bfloat16
    snn.readout_distill(z, ids, vals, lse, grad=view)  # written at those offsets
    assert near(view, b[2])


def _chain(V, student, u):
    ids, vals, lse = snn.readout_top(V, 4, 2.0)
    loss, row_loss, grad = snn.readout_distill(student, ids, vals, lse, 2.0)
    cls, logp, kept = snn.readout_sample(student, u)
    return ids, vals, lse, loss, row_loss, grad, cls, logp, kept


@pytest.mark.parametrize("C", [10, 100, 3001, 40001])
def test_streams_and_graphs(C):
    V, student, u = torch.randn((9, C), device="cuda"), torch.randn((9, C), device="cuda"), torch.rand(9, device="cuda")
    want = _chain(V, student, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _chain(V, student, u)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    from paper_2105_08810_amd import pipeline
    g = pipeline.Graphed(functools.partial(_chain, V, student, u))
    for k in range(4):
        V.copy_(torch.randn((9, C), device="cuda"))
        u.copy_(torch.rand(9, device="cuda"))
        got = [t.clone() for t in g()]
        want = _chain(V, student, u)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_binding_refuses():
    z = torch.zeros((4, 6), device="cuda")
    i, v = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    with pytest.raises(TypeError):
        snn.readout_top(z.double(), 2)
    with pytest.raises(ValueError):
        snn.readout_top(z.t(), 2)
    with pytest.raises(ValueError):
        snn.readout_top(z[0], 2)
    with pytest.raises(ValueError):
        snn.readout_top(z[:1].expand(4, 6), 2)
    with pytest.raises(snn.SnnError):
        snn.readout_top(z, 7)
    with pytest.raises(snn.SnnError):
        snn.readout_top(z, 2, tau=0.0)
    with pytest.raises(TypeError):
        snn.readout_distill(z, i.long(), v)
    with pytest.raises(ValueError):
        snn.readout_distill(z, i[:3], v)
    with pytest.raises(ValueError):
        snn.readout_distill(z, i, v, lse=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        snn.readout_distill(z, i, v, weight=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        snn.readout_distill(z, i, v, grad=torch.zeros((4, 7), device="cuda"))
    with pytest.raises(ValueError):
        snn.readout_distill(z, i, v, grad=torch.zeros((4, 6), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        snn.readout_sample(z, torch.zeros(3, device="cuda"))
    with pytest.raises(TypeError):
        snn.readout_sample(z, torch.zeros(4, device="cuda"), top_k=torch.zeros(4, device="cuda"))
    with pytest.raises(snn.SnnError):
        snn.readout_sample(torch.zeros((0, 6), device="cuda"), torch.zeros(0, device="cuda"))


# ---------------------------------------------------------------- many rows, where other kernels are taken than for few

MANY = [(300, 40, "normal", "f32"), (300, 100, "ties", "bf16"), (261, 128, "masked", "f16"), (300, 129, "normal", "bf16"),
        (300, 300, "lowest", "f32"), (270, 1000, "ties", "f16"), (270, 1000, "nan", "f32"), (257, 2100, "normal", "f32"),
        (257, 2100, "equal", "bf16"), (260, 5000, "peak", "f32"), (260, 9001, "normal", "bf16"), (258, 20000, "ties", "f32")]


@pytest.mark.parametrize("R,C,kind,dtype", MANY)
def test_many_rows_top(R, C, kind, dtype):
    view = _rows(_logits(np.random.default_rng(R + C), R, C, kind), dtype, C + C % 2, 0)
    for K in (3, 20):
        _check_top(_values(view), view, K, 2.0)


@pytest.mark.parametrize("R,C,kind,dtype", MANY)
def test_many_rows_sample(R, C, kind, dtype):
    rng = np.random.default_rng(R * C)
    view = _rows(_logits(rng, R, C, kind), dtype, C + C % 2, 0)
    some = slice(0, R) if C <= 300 else slice(0, R, 23)  # the oracle is a loop over classes
    settings = [None] * 4, _settings(rng, R, C), [_settings(rng, R, C)[0], None, _settings(rng, R, C)[2], None]
    u = rng.random(R).astype(np.float32)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    for t, k, p, m in settings:
        all_rows = [x.cpu().numpy() for x in snn.readout_sample(view, dev(u), dev(t), dev(k), dev(p), dev(m))]
        z = _values(view)[some]
        tt = (np.ones(R, np.float32) if t is None else t)[some]
        e = _e(z, tt)
        pick = lambda a, r, none: none if a is None else a[some][r]  # noqa: E731
        for r in range(len(z)):
            j, n, total, _ = rows.sample_row(z[r], e[r], u[some][r], int(pick(k, r, 0)), pick(p, r, 1.0),
                                             pick(m, r, 0.0), not tt[r] > 0)
            assert (all_rows[0][some][r], all_rows[2][some][r]) == (j, n), r
            if j >= 0:
                want = math.log(float(e[r, j]) * rows.UNIT / total)
                assert abs(all_rows[1][some][r] - want) <= U * 8 * (24 + abs(want))


@pytest.mark.parametrize("R,C,dtype", [(513, 130, "f32"), (513, 5000, "f32"), (513, 18001, "f32"), (512, 9000, "bf16"),
                                       (512, 17001, "bf16"), (513, 1500, "f16"), (20, 40000, "f32"), (3, 70001, "f16")])
def test_many_rows_distill(R, C, dtype):
    rng = np.random.default_rng(C)
    view = _rows(_logits(rng, R, C, "normal"), dtype)
    weight = rng.random(R).astype(np.float32)
    weight[::5] = 0.0
    rec = _record(rng, _values(view), 9, 1.5, "")
    _check_distill(view, *rec, 1.5, weight, dtype)
    full = torch.empty((R, C + 3), dtype=DTYPES[dtype], device="cuda")  # rows that begin otherwise than the logits'
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    a = snn.readout_distill(view, *map(dev, rec), 1.5, dev(weight))
    b = snn.readout_distill(view, *map(dev, rec), 1.5, dev(weight), grad=full[:, :C])
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_memory_is_the_given_streams(monkeypatch):
    """Outputs and workspaces of a call on a given stream are allocated on it: a workspace of another stream could be
    handed out there while the call still uses it."""
    side = torch.cuda.Stream()
    rng = np.random.default_rng(0)
    view = _rows(_logits(rng, 3, 70001, "normal"), "f32")  # shared among blocks: every call has a workspace
    u = torch.rand(3, device="cuda")
    weight, half = torch.ones(3, device="cuda"), torch.full((3,), 0.5, device="cuda")
    want = snn.readout_top(view, 20, 2.0), snn.readout_sample(view, u, weight, None, half, None)
    want += (snn.readout_distill(view, *want[0], 2.0, weight),)
    torch.cuda.synchronize()
    made, empty = [], torch.empty

    def counted(*a, **k):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(snn.torch, "empty", counted)
    got = (snn.readout_top(view, 20, 2.0, stream=side),
           snn.readout_sample(view, u, weight, None, half, None, stream=side))
    got += (snn.readout_distill(view, *got[0], 2.0, weight, stream=side),)
    monkeypatch.undo()
    side.synchronize()
    assert len(made) >= 3 + 1 + 3 + 1 + 3 + 1 and set(made) == {side.cuda_stream}
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("C,kind", [(129, "ties"), (130, "zeros"), (255, "wide"), (590, "ties"), (590, "lowest"),
                                    (1023, "normal"), (1302, "masked"), (2041, "ties"), (2048, "wide"), (2048, "equal"),
                                    (2049, "ties")])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_sample_cuts_of_middle_rows(C, kind, dtype):
    """Lengths that one wave holds and just beyond, top-k of every size, cuts within equal values, temperatures at which
    one weight or all of them count."""
    rng = np.random.default_rng(C)
    R = 40
    view = _rows(_logits(rng, R, C, kind), dtype, C + 5, C % 4)
    if kind == "lowest":
        view[view < -50000.0] = torch.finfo(DTYPES[dtype]).min
    temperature = (10.0 ** rng.uniform(-1.0, 1.0, R)).astype(np.float32)
    temperature[:4] = 1e-20, 1e30, 1e-5, 300.0
    top_k = rng.integers(2, C + 1, R).astype(np.int32)
    top_k[::7] = C - 1
    top_p = rng.random(R).astype(np.float32)
    top_p[::5] = 1.0
    top_p[1] = 0.0
    min_p = np.where(rng.random(R) < 0.5, 0.0, 0.05 * rng.random(R)).astype(np.float32)
    u = rng.random(R).astype(np.float32)
    for settings in ((top_k, None, None), (None, top_p, None), (top_k, top_p, min_p)):
        _check_sample(view, u, temperature, *settings)
