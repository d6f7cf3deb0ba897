"""The float64 oracle of the operators on rows of logits: gradients against differences, limits, closed forms."""
import math

import numpy as np
import pytest

from oracle import rows


@pytest.mark.parametrize("C,K,tau,tail", [(1, 1, 1.0, True), (2, 1, 2.0, True), (7, 3, 1.5, True), (7, 7, 0.5, True),
                                          (9, 4, 3.0, False), (40, 6, 1.0, True)])
def test_distill_gradient_is_the_differences(C, K, tau, tail):
    rng = np.random.default_rng(C * 10 + K)
    z = rng.normal(size=C) * 2
    teacher = rng.normal(size=(1, C)) * 2
    ids, vals, lse = rows.top(teacher, K, tau)
    one = (ids[0], vals[0], lse[0] if tail else None, tau)
    _, g, _, _ = rows.distill_row(z, *one)
    h = 1e-5
    for j in range(C):
        d = np.zeros(C)
        d[j] = h
        diff = (rows.distill_row(z + d, *one)[0] - rows.distill_row(z - d, *one)[0]) / (2 * h)
        # third derivatives of a log-sum-exp are below 1 / tau^3; rounding of a loss of size 1 below 1e-14 / h
        assert abs(diff - g[j]) <= h * h / tau ** 3 + 1e-8


def test_distill_of_all_classes_is_the_whole_divergence():
    rng = np.random.default_rng(0)
    z, t = rng.normal(size=12), rng.normal(size=(1, 12))
    p, q = np.exp(t[0] - rows.log_sum_exp(t[0])), np.exp(z - rows.log_sum_exp(z))
    for lse in (True, False):
        ids, vals, l = rows.top(t, 12, 1.0)
        loss, g, _, _ = rows.distill_row(z, ids[0], vals[0], l[0] if lse else None, 1.0)
        assert loss == pytest.approx(float((p * np.log(p / q)).sum()), rel=1e-12)
        assert np.allclose(g, q - p, atol=1e-14)
    # the teacher itself: nothing to learn
    ids, vals, l = rows.top(t, 5, 1.0)
    loss, g, _, _ = rows.distill_row(t[0], ids[0], vals[0], l[0], 1.0)
    assert abs(loss) < 1e-14 and np.abs(g).max() < 1e-14


def test_distill_empty_rows():
    z = np.array([0.5, -1.0, 2.0])
    none = np.array([-1, -1])
    for lse in (None, 3.0):  # with a log-sum-exp all of the teacher is on the other classes, which are all classes
        loss, g, _, _ = rows.distill_row(z, none, np.array([-np.inf, -np.inf]), lse, 1.0)
        assert abs(loss) < 1e-15 and np.abs(g).max() < 1e-15
    loss, g, _, _ = rows.distill_row(np.full(3, -np.inf), np.array([1]), np.array([0.3]), None, 1.0)
    assert loss == math.inf and np.array_equal(g, [0.0, -1.0, 0.0])


def test_top_order_and_padding():
    z = np.array([[1.0, 3.0, 3.0, np.nan, -np.inf, 0.0, -0.0]])
    ids, vals, lse = rows.top(z, 6, 1.0)
    assert ids[0].tolist() == [1, 2, 0, 5, 6, -1]
    assert vals[0].tolist() == [3.0, 3.0, 1.0, 0.0, 0.0, -np.inf]
    assert lse[0] == pytest.approx(math.log(2 * math.exp(3) + math.exp(1) + 2))


def test_sample_filters():
    z = np.log(np.array([4.0, 2.0, 1.0, 1.0, 8.0]))
    e = (np.exp(z - z.max())).astype(np.float32)

    def classes(**kw):
        return {rows.sample_row(z, e, u, **kw)[0] for u in np.linspace(0, 0.9999, 400)}

    assert classes() == {0, 1, 2, 3, 4}
    assert classes(top_k=2) == {0, 4}
    assert classes(top_k=4) == {0, 1, 2, 4}  # of two equal classes the first
    assert classes(top_p=0.5) == {4}  # 8 of 16 reach one half
    assert classes(top_p=0.51) == {0, 4}
    assert classes(min_p=0.25) == {0, 1, 4}
    assert classes(greedy=True) == {4}
    assert rows.sample_row(z, e, 0.0)[0] == 0 and rows.sample_row(z, e, 1.0)[0] == 4
    assert rows.sample_row(np.full(4, -np.inf), np.zeros(4, np.float32), 0.5)[0] == -1
    # with the probabilities 4 2 1 1 8 of 16, u in [i/16, (i+1)/16) is the i-th sixteenth in the order of the classes
    want = [0] * 4 + [1] * 2 + [2] + [3] + [4] * 8
    e = np.array([0.5, 0.25, 0.125, 0.125, 1.0], np.float32)
    assert [rows.sample_row(z, e, (i + 0.5) / 16)[0] for i in range(16)] == want


def test_distill_does_not_see_a_common_shift():
    """A row and a teacher without a log-sum-exp shifted by a number that their logits are small beside."""
    rng = np.random.default_rng(4)
    z, ids, vals = np.round(rng.normal(size=9) * 64) / 64, np.array([5, 0, 7]), np.round(rng.normal(size=3) * 64) / 64
    want = rows.distill_row(z, ids, vals, None, 1.5)
    for by in (1024.0, -2.0 ** 40):
        for got in (rows.distill_row(z + by, ids, vals, None, 1.5), rows.distill_row(z, ids, vals + by, None, 1.5)):
            assert got[0] == pytest.approx(want[0], rel=1e-12) and np.allclose(got[1], want[1], rtol=1e-12, atol=1e-15)
    lowest = float(np.finfo(np.float32).min)
    loss, g, _, _ = rows.distill_row(np.full(4, lowest), np.array([1]), np.array([0.3]), None, 1.0)
    assert loss == pytest.approx(math.log(4)) and np.allclose(g, [0.25, -0.75, 0.25, 0.25])
    loss, g, _, _ = rows.distill_row(np.zeros(4), np.array([1, 2]), np.full(2, lowest), None, 1.0)
    assert loss == pytest.approx(math.log(2)) and np.allclose(g, [0.25, -0.25, -0.25, 0.25])
    z = np.array([0.5, lowest, lowest, lowest, 1.0])  # the classes not listed, all at the lowest value, share alike
    _, g, _, share = rows.distill_row(z, np.array([0, 4]), np.array([0.0, 0.0]), 2.0, 1.0)
    p_t = 1 - 2 * math.exp(-2)
    assert np.allclose(share, [0, 1 / 3, 1 / 3, 1 / 3, 0]) and np.allclose(g[1:4], -p_t / 3)
    z = np.array([0.5, 1.0, -lowest])  # beside the highest value too
    _, g, _, share = rows.distill_row(z, np.array([2]), np.array([0.0]), 2.0, 1.0)
    assert np.allclose(share[:2], np.exp([0.5, 1.0]) / np.exp([0.5, 1.0]).sum())
