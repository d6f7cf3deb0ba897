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


# ---------------------------------------------------------------- logits at the ends of a type's range

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ENDS = ["lowest", "one above", "few", "highest", "both", "far"]


def _ends(rng, R, C, dtype, kind):
    """Rows with the type's lowest or highest value, as a mask or an overflow leaves them."""
    info = torch.finfo(DTYPES[dtype])
    z = torch.from_numpy((rng.standard_normal((R, C)) * 2).astype(np.float32))
    if kind in ("lowest", "one above"):
        z[:] = info.min
    if kind == "one above":
        z[:, C // 2] = -1.0
    if kind == "few":  # some at the lowest value, no other class possible
        z[:] = -INF
        z[:, ::max(1, C // 300)] = info.min
    if kind in ("highest", "both"):
        z[:, C // 3] = info.max
        z[:, C - 1] = info.max
    if kind == "both":
        z[:, : C // 3] = info.min
    if kind == "far":  # no end of the range, and yet a product with 1 / tau is rounded by more than a row's sum spans
        z *= info.max ** 0.3
    return z.to(DTYPES[dtype]).cuda()


# lengths of every kernel: 16 lanes a row, one wave, blocks with rows in registers, few long rows in parts, passes
END_LENGTHS = [1, 10, 100, 128, 129, 700, 2048, 2049, 5000, 20000, 40000, 70001]


@pytest.mark.parametrize("kind", ENDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", END_LENGTHS)
def test_record_at_the_ends_of_the_range(C, dtype, kind):
    view = _ends(np.random.default_rng(C), 3, C, dtype, kind)
    z = view.float().cpu().numpy()
    for tau in (0.5, 1.0, 1.7, 4.0):
        K = min(C, 6)
        ids, vals, lse = snn.readout_top(view, K, tau)
        i, v, _ = rows.top(z, K, tau)
        assert np.array_equal(ids.cpu().numpy(), i) and np.array_equal(vals.cpu().numpy().astype(np.float64), v)
        got = lse.cpu().numpy().astype(np.float64)
        for r in range(len(z)):
            x = z[r].astype(np.float64)
            m = x.max()
            want = m / tau + math.log(np.exp((x - m) / tau).sum())
            if abs(want) > float(np.finfo(np.float32).max):  # beyond float32
                assert got[r] == math.copysign(INF, want)
            else:  # the quotient's two roundings, the sum's additions, a logarithm below log C, the last addition
                assert abs(got[r] - want) <= U * (4 * abs(m) / tau + 8 * (1 + math.log(C)) + C / 1024 + 86), (r, tau)


# ---------------------------------------------------------------- distillation where some logits are not finite

# relative rounding of a result to its type, and the spacing of its smallest numbers
ROUND = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 2.0 ** -133), "f16": (2.0 ** -11, 2.0 ** -25)}
# lengths of every kernel: 16 lanes a row, one wave, blocks, rows read twice
DISTILL_LENGTHS = [3, 20, 100, 300, 1500, 5000, 12000, 30000, 70001, 140003]


def _device(*arrays):
    return [None if a is None else torch.from_numpy(a).cuda() for a in arrays]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", DISTILL_LENGTHS)
def test_listed_classes_that_cannot_be_given(C, dtype):
    """All listed logits are -inf and the others lie far below 0: the listed ones' gradient is -p / tau, the others' the
    student's share of them."""
    rng = np.random.default_rng(C)
    z = rng.standard_normal((4, C)).astype(np.float32) + np.array([[-100.0], [-1000.0], [-30000.0], [0.0]], np.float32)
    ids = np.stack([rng.choice(C, 2, replace=False) for _ in range(4)]).astype(np.int32)
    np.put_along_axis(z, ids, -INF, 1)
    view = torch.from_numpy(z).to(DTYPES[dtype]).cuda()
    z = view.float().cpu().numpy()
    vals = rng.standard_normal((4, 2)).astype(np.float32)
    lse = (2.0 + rng.random(4)).astype(np.float32)
    for tau, tail in ((1.0, False), (2.0, True)):
        l = lse if tail else None
        _, _, want, env, share = rows.distill(z, ids, vals, l, tau)
        _, row_loss, grad = snn.readout_distill(view, *_device(ids, vals, l), tau)
        got = grad.double().cpu().numpy()
        assert bool((row_loss == INF).all())
        # float32 sums, exponents of size below A formed in a few roundings, and p_t's error by each class's share
        A = np.array([104.0, 1004.0, 30004.0, 4.0])[:, None] / tau + 4
        rel = U * (102 + C / 1024 + 6 * A)
        out, tiny = ROUND[dtype]
        tol = rel * (env + share / tau) + tiny
        assert (np.abs(got - want) <= tol + out * (np.abs(want) + tol)).all(), (tau, tail)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", DISTILL_LENGTHS)
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_one_value_makes_the_rows_gradient_nan(C, dtype, what):
    """A NaN or +inf among finite logits, among masked ones and alone with them, at a listed class and at another: the
    row's loss and all of its gradient are NaN, the rows beside it are as they are without it."""
    rng = np.random.default_rng(C + 1)
    kinds = [(fill, listed) for fill in ("finite", "masked", "others masked") for listed in (False, True)]
    R = len(kinds) + 1  # the last row stays whole
    z = rng.standard_normal((R, C)).astype(np.float32)
    ids = np.stack([rng.choice(C, 2, replace=False) for _ in range(R)]).astype(np.int32)
    for r, (fill, listed) in enumerate(kinds):
        other = next(j for j in range(C) if j not in ids[r])
        if fill == "masked":
            z[r] = -INF
        elif fill == "others masked":
            keep = z[r, ids[r]].copy()
            z[r] = -INF
            z[r, ids[r]] = keep
        z[r, ids[r, 0] if listed else other] = np.nan if what == "nan" else INF
    view = torch.from_numpy(z).to(DTYPES[dtype]).cuda()
    vals = rng.standard_normal((R, 2)).astype(np.float32)
    lse = (2.0 + rng.random(R)).astype(np.float32)
    for tail in (False, True):
        for into in (False, True):
            start = torch.ones((R, C), dtype=DTYPES[dtype], device="cuda") if into else None
            dev = _device(ids, vals, lse if tail else None)
            _, row_loss, grad = snn.readout_distill(view, *dev, 1.5, grad=start, accumulate=into)
            assert bool(row_loss[:-1].isnan().all()) and bool(row_loss[-1:].isfinite().all())
            assert bool(grad[:-1].isnan().all()) and bool(grad[-1:].isfinite().all())
            assert bool(row_loss[-1] == snn.readout_distill(view[-1:], *(None if t is None else t[-1:] for t in dev), 1.5)[1][0])


def _ends_of_distill(rng, C, info):
    """Rows at and near the ends of a type's range, by name, with the classes that are listed."""
    far = float(info.max) ** 0.3
    k = rng.choice(C, 2, replace=False)
    plain = rng.standard_normal(C).astype(np.float32)
    out = {}
    for name, mask in (("lowest", info.min), ("masked", max(-1e9, info.min)), ("far", -far)):
        z = np.full(C, mask, np.float32)
        out[name] = z, k
        out[name + ", listed not"] = np.where(np.isin(np.arange(C), k), plain, z), k
        out[name + " listed"] = np.where(np.isin(np.arange(C), k), z, plain), k
        z = z.copy()
        z[[j for j in range(C) if j not in k][0]] = 0.5
        out[name + ", one not"] = z, k
    z = plain.copy()
    z[k[0]] = info.max
    out["highest listed"] = z, k
    z = plain.copy()
    z[[j for j in range(C) if j not in k][0]] = info.max
    out["highest"] = z, k
    out["all far"] = (plain * far).astype(np.float32), k
    out["shifted"] = (plain + 2000.0).astype(np.float32), k
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", DISTILL_LENGTHS)
def test_distill_at_the_ends_of_the_range(C, dtype):
    rng = np.random.default_rng(C + 2)
    cases = _ends_of_distill(rng, C, torch.finfo(DTYPES[dtype]))
    names = list(cases)
    view = torch.from_numpy(np.stack([cases[n][0] for n in names])).to(DTYPES[dtype]).cuda()
    ids = np.stack([cases[n][1] for n in names]).astype(np.int32)
    z = view.float().cpu().numpy()
    R = len(names)
    vals = rng.standard_normal((R, 2)).astype(np.float32)
    lse = (2.0 + rng.random(R)).astype(np.float32)
    lowest = np.full((R, 2), np.finfo(np.float32).min, np.float32)  # a teacher's row at the lowest value
    for tau, v, l in ((1.0, vals, lse), (2.5, vals, None), (1.0, lowest, None), (1.0, vals - np.float32(1e7), None)):
        _, row_loss, grad = snn.readout_distill(view, *_device(ids, v, l), tau)
        got_l, got = row_loss.double().cpu().numpy(), grad.double().cpu().numpy()
        with np.errstate(over="ignore"):
            _, want_l, want, env, share = rows.distill(z, ids, v, l, tau)
        for r in range(R):
            x = z[r].astype(np.float64) / tau
            m = x.max()
            logq = x - m - math.log(np.exp(x - m).sum())
            logp = v[r].astype(np.float64) / tau
            logp = logp - l[r] if l is not None else logp - logp.max() - math.log(np.exp(logp - logp.max()).sum())
            p = np.exp(logp)
            other = np.ones(C, bool)
            other[ids[r]] = False
            logq_t = logq[other].max() + math.log(np.exp(logq[other] - logq[other].max()).sum())
            p_t = max(0.0, 1 - p.sum()) if l is not None else 0.0
            terms = (p * (np.abs(logp) + np.abs(logq[ids[r]]))).sum() + (p_t * (abs(math.log(p_t)) + abs(logq_t)) if p_t else 0)
            # float32 sums, exponents and logarithms of numbers of size A in a few roundings; p_t = 1 - sum p
            A = (abs(m) if abs(m) < 1024 else 0) + np.abs(logp).max() + (np.abs(v[r]).max() / tau if np.abs(v[r]).max() < 1024 else 0)
            rel = U * (102 + C / 1024 + 8 * A)
            tol = rel * (1 + terms) + (rel * (abs(logq_t) + abs(math.log(p_t)) + 1) if p_t else 0)
            if abs(want_l[r]) > np.finfo(np.float32).max:
                assert got_l[r] == INF, names[r]
            else:
                assert abs(got_l[r] - want_l[r]) <= tol, (names[r], tau, got_l[r], want_l[r])
            out, tiny = ROUND[dtype]
            tol = rel * (env[r] + 4 * share[r] * (l is not None) / (R * tau)) + tiny + 2.0 ** -126
            bad = ~(np.abs(got[r] - want[r]) <= tol + out * (np.abs(want[r]) + tol))
            assert not bad.any(), (names[r], tau, np.flatnonzero(bad)[:4], got[r][bad][:4], want[r][bad][:4])


# ---------------------------------------------------------------- more rows than one launch counts

def _some_rows(R):
    """Rows at the ends, at where one launch may end and another begin, and between."""
    at = {0, 1, R - 1, R // 2}
    for k in range(10, 32):
        at |= {(1 << k) - 1, 1 << k, (1 << k) + 1}
    return sorted(r for r in at if r < R)


@pytest.mark.parametrize("R,C", [((1 << 28) + 5, 1), ((1 << 26) + 5, 129)])
def test_more_rows_than_a_launch_counts(R, C):
    """Threads of a dispatch are counted in 32 bits: 16 a row of one class, 64 a row of 129 pass that. Every row is what it
    is in a call of its own."""
    g = torch.Generator(device="cuda").manual_seed(C)
    z = torch.empty((R, C), dtype=torch.bfloat16, device="cuda")
    for part in z.split(1 << 24):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda", dtype=torch.bfloat16))
    at = _some_rows(R)
    K = min(C, 2)
    ids, vals, lse = snn.readout_top(z, K, 2.0)
    for r in at:
        for a, b in zip((ids, vals, lse), snn.readout_top(z[r:r + 1], K, 2.0)):
            assert torch.equal(a[r:r + 1], b), r
    if C == 1:
        assert bool((ids == 0).all()) and torch.equal(vals.view(-1), z.view(-1).float())
    loss, row_loss, grad = snn.readout_distill(z, ids, vals, lse, 1.0)
    one = torch.full((1,), 1.0 / R, device="cuda")  # the mean's weight, rounded to float32
    assert abs(float(loss) - float(row_loss.double().sum() * one.double())) <= U * abs(float(loss)) + 1e-9
    for r in at:
        alone = snn.readout_distill(z[r:r + 1], ids[r:r + 1], vals[r:r + 1], lse[r:r + 1], 1.0, one)
        assert torch.equal(row_loss[r:r + 1], alone[1]) and torch.equal(grad[r:r + 1], alone[2]), r
    del ids, vals, lse, row_loss, grad
    u = torch.rand(R, generator=g, device="cuda")
    p = torch.full((R,), 0.7, device="cuda")
    cls, logp, kept = snn.readout_sample(z, u, None, None, p)
    for r in at:
        for a, b in zip((cls, logp, kept), snn.readout_sample(z[r:r + 1], u[r:r + 1], None, None, p[r:r + 1])):
            assert torch.equal(a[r:r + 1], b), r


# ---------------------------------------------------------------- the highest temperatures

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [5, 20, 100, 700, 2048, 3000, 12000, 40000, 140003])
def test_draws_at_the_highest_temperatures(C, dtype):
    """Up to the largest float32 a temperature is what it says, masks of the type's lowest value included, and beyond it all
    finite logits are alike."""
    temperature = np.array([1e29, 1e31, 1e36, 2e37, 1e38, 3e38, INF, INF], np.float32)
    R = len(temperature)
    rng = np.random.default_rng(C)
    z = rng.standard_normal((R, C)).astype(np.float32) * 3
    z[rng.random((R, C)) < 0.4] = torch.finfo(DTYPES[dtype]).min
    z[rng.random((R, C)) < 0.1] = -INF
    z[:, C // 2] = 1.0
    view = torch.from_numpy(z).to(DTYPES[dtype]).cuda()
    x = view.float()
    m = x.amax(1, keepdim=True)
    t = torch.where(x == m, torch.zeros_like(x), (x - m) * (1.0 / torch.from_numpy(temperature).cuda()[:, None]))
    e = torch.where(x > -INF, torch.exp(t), torch.zeros_like(x)).cpu().numpy()
    x = x.cpu().numpy()
    u = rng.random(R).astype(np.float32)
    top_k = rng.integers(1, C + 1, R).astype(np.int32)
    top_p = (0.5 + 0.5 * rng.random(R)).astype(np.float32)
    for k, p in ((None, None), (top_k, None), (None, top_p), (top_k, top_p)):
        cls, logp, kept = (v.cpu().numpy() for v in snn.readout_sample(view, *_device(u, temperature, k, p)))
        for r in range(R):
            j, n, total, own = rows.sample_row(x[r], e[r], u[r], 0 if k is None else int(k[r]), 1.0 if p is None else p[r])
            assert (cls[r], kept[r]) == (j, n), (temperature[r], k is None, p is None)
            want = math.log(own / total)  # as a drawn weight is within 2^-32 of its e
            assert abs(logp[r] - want) <= U * 8 * (24 + abs(want))


# ---------------------------------------------------------------- the longest rows, and ways that few calls take

def _long_rows(rng, C, lead, dtype, kind):
    z = (rng.standard_normal((1, C)) * 2.5).astype(np.float32)
    if kind == "ties":
        z = np.round(z)
    full = torch.full((C + lead,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    view = full[lead:].view(1, C)
    view.copy_(torch.from_numpy(z))
    return view, view.float().cpu().numpy()


LONGEST = [(1 << 20, 0, "f32", "normal"), ((1 << 20) - 1, 1, "bf16", "ties"), (1 << 20, 3, "f16", "normal"),
           (300001, 1, "f32", "ties"), (600003, 3, "bf16", "normal")]


@pytest.mark.parametrize("C,lead,dtype,kind", LONGEST)
def test_longest_records(C, lead, dtype, kind):
    view, z = _long_rows(np.random.default_rng(C + lead), C, lead, dtype, kind)
    for K in (1, 60, 1024):
        ids, vals, lse = snn.readout_top(view, K, 1.5)
        i, v, l = rows.top(z, K, 1.5)
        assert np.array_equal(ids.cpu().numpy(), i) and np.array_equal(vals.cpu().numpy().astype(np.float64), v)
        # a thread's share of the additions, a tree, and the roundings around them
        assert abs(float(lse[0]) - l[0]) <= U * (4 * np.abs(z).max() / 1.5 + 8 * (1 + math.log(C)) + C / 1024 + 86)


@pytest.mark.parametrize("C,lead,dtype,kind", LONGEST)
def test_longest_distillation(C, lead, dtype, kind):
    rng = np.random.default_rng(C + lead)
    view, z = _long_rows(rng, C, lead, dtype, kind)
    ids, vals, lse = rows.top((0.7 * z + rng.standard_normal(z.shape)).astype(np.float32), 200, 1.5)
    rec = ids.astype(np.int32), vals.astype(np.float32), lse.astype(np.float32)
    for tail in (True, False):
        r = rec[0], rec[1], rec[2] if tail else None
        loss, row_loss, grad = snn.readout_distill(view, *_device(*r), 1.5)
        lo, _, want, env, share = rows.distill(z, *r, 1.5)
        A = (np.abs(z).max() + np.abs(rec[1]).max()) / 1.5 + 1
        rel = U * (102 + C / 1024 + 200 / 64 + 6 * A)
        assert abs(float(row_loss[0]) - lo) <= rel * (1 + 2 * A) + (rel * (2 + 2 * A) if tail else 0)
        assert float(loss[0]) == float(row_loss[0])
        out, tiny = ROUND[dtype]
        tol = rel * (env + 4 * share * tail / 1.5) + tiny
        got = grad.double().cpu().numpy()
        assert (np.abs(got - want) <= tol + out * (np.abs(want) + tol) * 1.01 + 2.0 ** -126).all()


@pytest.mark.parametrize("C,lead,dtype,kind", LONGEST)
def test_longest_draws(C, lead, dtype, kind):
    rng = np.random.default_rng(C + lead)
    view, z = _long_rows(rng, C, lead, dtype, kind)
    x = view.float()
    for k, p, temperature, u in ((0, 1.0, 1.0, 0.61), (0, 0.9, 0.7, 0.3), (700, 0.95, 1.3, 0.97), (5, 1.0, 1.0, 0.5),
                                 (1, 1.0, 1.0, 0.2)):
        t = torch.full((1,), temperature, device="cuda")
        m = x.amax(1, keepdim=True)
        e = torch.exp(torch.where(x == m, torch.zeros_like(x), (x - m) * (1.0 / t[:, None]))).cpu().numpy()
        cls, logp, kept = snn.readout_sample(view, torch.full((1,), u, device="cuda"), t,
                                             torch.full((1,), k, dtype=torch.int32, device="cuda"),
                                             torch.full((1,), p, device="cuda"))
        j, n, total, own = rows.sample_row(z[0], e[0], np.float32(u), k, np.float32(p))
        assert (int(cls[0]), int(kept[0])) == (j, n), (k, p)
        assert abs(float(logp[0]) - math.log(own / total)) <= U * 8 * (24 + abs(math.log(own / total)))


@pytest.mark.parametrize("R,C,K", [(3, 5000, 600), (3, 4096, 1000), (2, 9001, 1024)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_records_of_many_classes_of_middle_rows(R, C, K, dtype):
    rng = np.random.default_rng(C + K)
    view = torch.from_numpy((rng.standard_normal((R, C)) * 2).astype(np.float32)).to(DTYPES[dtype]).cuda()
    i, v, _ = rows.top(view.float().cpu().numpy(), K, 1.0)
    ids, vals, _ = snn.readout_top(view, K, 1.0)
    assert np.array_equal(ids.cpu().numpy(), i) and np.array_equal(vals.cpu().numpy().astype(np.float64), v)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R", [3, 700])
@pytest.mark.parametrize("C", [20, 120, 1000, 5000, 18000, 70001])
def test_loss_without_a_gradient_is_the_same(R, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(C)
    z = torch.randn((R, C), generator=g, device="cuda").to(DTYPES[dtype])
    rec = snn.readout_top(z.float() + torch.randn((R, C), generator=g, device="cuda"), 4, 2.0)
    weight = torch.rand(R, generator=g, device="cuda")
    weight[::5] = 0.0
    with_grad, without = snn.readout_distill(z, *rec, 2.0, weight), snn.readout_distill(z, *rec, 2.0, weight, want_grad=False)
    assert without[2] is None and torch.equal(with_grad[0], without[0]) and torch.equal(with_grad[1], without[1])


# ---------------------------------------------------------------- where one way ends and another begins

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C,lead", [(1, 65536, 0), (2, 65536, 1), (2, 98303, 0), (2, 98304, 3), (128, 98304, 0), (129, 98304, 0),
                                      (2, 131072, 0), (130, 131071, 1), (3, 16384, 0), (3, 16385, 1), (63, 32768, 0),
                                      (64, 32768, 0), (64, 32761, 5)])
def test_records_where_ways_change(R, C, lead, dtype):
    g = torch.Generator(device="cuda").manual_seed(C)
    full = torch.randn(R * C + lead, generator=g, device="cuda").to(DTYPES[dtype])
    z = full[lead:].view(R, C)
    x = z.float()
    for K in (3, 100):
        ids, vals, lse = snn.readout_top(z, K, 2.0)
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        assert torch.equal(ids, i[:, :K].to(torch.int32)) and torch.equal(vals, v[:, :K])
        # logits below 8: two roundings of the quotient, a logarithm below 12, a thread's additions and a tree
        assert float((lse.double() - torch.logsumexp(x.double() / 2.0, 1)).abs().max()) <= U * (16 + 8 * 13 + 128 + 86)


def test_graph_of_rows_shared_among_blocks():
    z, u = torch.randn((5, 140001), device="cuda"), torch.rand(5, device="cuda")
    call = lambda: (*snn.readout_top(z, 40, 1.5), *snn.readout_sample(z, u, top_p=torch.full_like(u, 0.9)))  # noqa: E731
    call()
    g = pipeline.Graphed(call)
    for _ in range(3):
        z.copy_(torch.randn_like(z))
        u.copy_(torch.rand_like(u))
        got, want = [t.clone() for t in g()], call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,C", [(3, 1025), (3, 4097), (256, 4100), (257, 4100), (3, 16384), (3, 16385), (257, 16384), (3, 32768),
                                 (3, 32769), (3, 65536), (3, 65537), (64, 128), (65, 128), (64, 129)])
def test_distillation_where_ways_change(R, C, dtype):
    """Against the formula in 64 bits on the device."""
    g = torch.Generator(device="cuda").manual_seed(R + C)
    z = (torch.randn((R, C), generator=g, device="cuda") * 2).to(DTYPES[dtype])
    K, tau = 9, 1.5
    ids, vals, lse = snn.readout_top(z.float() * 0.7 + torch.randn((R, C), generator=g, device="cuda"), K, tau)
    at = ids.long()
    logq = torch.log_softmax(z.double() / tau, 1)
    logp = vals.double() / tau - lse.double()[:, None]
    p = torch.exp(logp)
    left = (1 - p.sum(1)).clamp_min(0)
    others = torch.exp(logq).scatter(1, at, 0.0)
    q_t = others.sum(1)
    want = (p * (logp - logq.gather(1, at))).sum(1) + left * (torch.log(left) - torch.log(q_t))
    target = (others * (left / q_t)[:, None]).scatter(1, at, p)
    grad = (torch.exp(logq) - target) / (tau * R)
    loss, row_loss, got = snn.readout_distill(z, ids, vals, lse, tau)
    # float32 sums and exponents of numbers of size A; p_t = 1 - sum p, which goes to the others by their share
    A = float(z.float().abs().max() + vals.abs().max()) / tau + math.log(C)
    rel = U * (102 + C / 1024 + 6 * A)
    assert bool(((row_loss.double() - want).abs() <= rel * (4 + 4 * A)).all())
    assert abs(float(loss) - float(want.mean())) <= rel * (4 + 4 * A)
    out, tiny = ROUND[dtype]
    tol = rel * (torch.exp(logq) + target + 4 * others / q_t[:, None]) / (tau * R) + tiny
    assert bool(((got.double() - grad).abs() <= tol + out * (grad.abs() + tol)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [33, 48, 49, 64, 100, 128])
def test_draws_where_ways_change(C, dtype):
    """Rows drawn in calls of many and of few rows, with and without an order, have the same answers."""
    R = 100 * (C - 32) + 3
    g = torch.Generator(device="cuda").manual_seed(C)
    z = (torch.randn((R, C), generator=g, device="cuda") * 2).round(decimals=1).to(DTYPES[dtype])
    u = torch.rand(R, generator=g, device="cuda")
    k = torch.randint(0, C + 1, (R,), generator=g, device="cuda", dtype=torch.int32)
    p, m = torch.rand(R, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda") * 0.1
    t = torch.rand(R, generator=g, device="cuda") * 2
    for settings in ((t, k, p, m), (t, None, p, None), (None, k, None, None), (t, None, None, m)):
        whole = snn.readout_sample(z, u, *settings)
        for part in (slice(0, 40), slice(R - 41, R)):
            few = snn.readout_sample(z[part], u[part], *(None if s is None else s[part] for s in settings))
            assert all(torch.equal(a[part], b) for a, b in zip(whole, few))
    e = torch.exp((z.float() - z.float().amax(1, keepdim=True)) * (1.0 / torch.ones((R, 1), device="cuda"))).cpu().numpy()
    x = z.float().cpu().numpy()
    cls, _, kept = snn.readout_sample(z, u, None, k, None)
    for r in range(0, R, 97):
        assert (int(cls[r]), int(kept[r])) == rows.sample_row(x[r], e[r], u[r].cpu().numpy(), int(k[r]))[:2]
